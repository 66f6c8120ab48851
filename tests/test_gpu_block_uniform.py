"""GPU: block-scaled products against the per-tensor product, and against themselves.

Where all scales of an operand are one power of two, the per-tensor product of the same codes computes the same sums in the same order and
multiplies the same power of two in at the end.  Powers of two move no rounding (everything here stays far from binary32's ends), so that
the two agree bit for bit: what a block-scaled product rounds is what the matrix instruction rounds, and nothing more."""
import numpy as np
import pytest
import torch

from oracle import gemm
from paper_2505_20524_amd import fog

pytestmark = pytest.mark.gpu

LAYOUTS = [gemm.NT, gemm.NN, gemm.TN]
SIZES = [(2048, 8192, 1040), (1744, 2480, 9296), (1776, 3088, 2064), (2560, 1024, 4112), (4112, 4064, 528), (1040, 2064, 784), (272, 272, 9232), (304, 272, 400)]


def codes(rng, *shape):
    return torch.from_numpy((rng.integers(0, 0x70, shape) | rng.integers(0, 2, shape) << 7).astype(np.uint8)).cuda()


def stored(layout, M, N, K):
    return ((K, M) if layout == gemm.TN else (M, K)), ((N, K) if layout == gemm.NT else (K, N))


def room(layout, M, N, K):
    return torch.empty(max(fog.fp8_gemm_workspace(layout, M, N, K), 16), dtype=torch.uint8, device="cuda")


def scales(shape, kind, i, blocks, byte):
    shape = tuple(-(-n // 128) for n in shape) if kind == fog.TILE else (blocks, i)
    return torch.full(shape, byte, dtype=torch.uint8, device="cuda")


@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("M,N,K", SIZES)
@pytest.mark.parametrize("kind_a,kind_b", [(fog.VECTOR, fog.TILE), (fog.TILE, fog.VECTOR)])
def test_equal_scales_give_the_per_tensor_product(layout, M, N, K, kind_a, kind_b):
    rng = np.random.default_rng(M + N + K)
    sh_a, sh_b = stored(layout, M, N, K)
    A, B, ws = codes(rng, *sh_a), codes(rng, *sh_b), room(layout, M, N, K)
    ea, eb, blocks = 119, 131, -(-K // 128)
    C, D = (torch.full((M, N), v, dtype=torch.bfloat16, device="cuda") for v in (3.0, 5.0))
    fog.fp8_gemm_block(layout, M, N, K, A, fog.E4M3, kind_a, scales(sh_a, kind_a, M, blocks, ea), B, fog.E4M3, kind_b, scales(sh_b, kind_b, N, blocks, eb), C, workspace=ws)
    sinv = [torch.tensor([2.0 ** (e - 127)], device="cuda") for e in (ea, eb)]
    fog.fp8_gemm(layout, M, N, K, A, fog.E4M3, sinv[0], B, fog.E4M3, sinv[1], D, workspace=ws)
    assert torch.equal(C.view(torch.int16), D.view(torch.int16))


@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("M,N,K", SIZES + [(1, 4096, 4096), (24, 2064, 4112), (32, 4096, 1040)])
def test_a_product_is_the_same_on_every_run(layout, M, N, K):
    rng = np.random.default_rng(M * 3 + N + K)
    if layout == gemm.TN and M % 16:
        M = 16
    sh_a, sh_b = stored(layout, M, N, K)
    A, B, ws = codes(rng, *sh_a), codes(rng, *sh_b), room(layout, M, N, K)
    sa, sb = (torch.from_numpy(rng.integers(110, 140, (-(-K // 128), n)).astype(np.uint8)).cuda() for n in (M, N))
    first = None
    for fill in (0.0, 1.0, float("nan"), 2.0, 3.0, 4.0):
        C = torch.full((M, N), fill, dtype=torch.bfloat16, device="cuda")
        ws.fill_(0xFF if first is None else 0)
        fog.fp8_gemm_block(layout, M, N, K, A, fog.E4M3, fog.VECTOR, sa, B, fog.E4M3, fog.VECTOR, sb, C, workspace=ws)
        first = C if first is None else first
        assert torch.equal(C.view(torch.int16), first.view(torch.int16))
    assert bool(torch.isfinite(first).all())
