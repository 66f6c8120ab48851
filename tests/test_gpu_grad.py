"""GPU parity: the global norm of gradients and their clipping, against float64."""
import math

import numpy as np
import pytest
import torch

from paper_2505_20524_amd import fog

pytestmark = pytest.mark.gpu

FLT_MAX = float(np.finfo(np.float32).max)


def norm_of(grads):
    jobs = fog.make_grad_jobs([(g, g) for g in grads])
    sumsq = torch.full((1,), -1.0, dtype=torch.float64, device="cuda")
    ws = torch.full((max(fog.grad_sumsq_workspace(len(grads)), 8),), 0xFF, dtype=torch.uint8, device="cuda")
    fog.grad_sumsq(jobs, sumsq, ws)
    return jobs, sumsq


def exact_sumsq(grads):
    return math.fsum(float((g.double() ** 2).sum()) for g in grads)


def check_clip(grads, max_norm, outs=None):
    """One norm and one clip, in place or to `outs`."""
    before = [g.clone() for g in grads]
    total = exact_sumsq(grads)
    _, sumsq = norm_of(grads)
    jobs = fog.make_grad_jobs(list(zip(grads, outs)) if outs else list(grads))
    norm = torch.zeros(1, device="cuda")
    fog.grad_clip(jobs, sumsq, max_norm, norm)
    torch.cuda.synchronize()
    n = sum(g.numel() for g in grads)
    # binary64 sums of n squares in any order, on both sides
    assert abs(sumsq.item() - total) <= 2 * (n + 2) * 2.0 ** -53 * total
    r = math.sqrt(total)
    # a finite norm beyond binary32 (9.5e39 in one test below; the largest binary32 is 3.4e38) is told as the largest finite number
    assert norm.item() == FLT_MAX if r > FLT_MAX else abs(norm.item() - r) <= (2.0 ** -24 + (n + 4) * 2.0 ** -53) * r
    c = max_norm / r if r > max_norm else 1.0
    for b, g, o in zip(before, grads, outs or grads):
        want = b.double() * c
        # the factor and the product in binary32, then half a step of the type; binary32 results below the normal range by a whole step of it
        tol = (2 * 2.0 ** -24 + (n + 4) * 2.0 ** -53 + torch.finfo(b.dtype).eps / 2) * 1.01 * want.abs() + (2.0 ** -149 if c != 1.0 else 0.0)
        tol = tol + (2.0 ** -133 if c != 1.0 and b.dtype == torch.bfloat16 else 0.0)
        assert bool(((o.double() - want).abs() <= tol).all())
        if outs:
            assert torch.equal(b, g)
        if c == 1.0:
            assert torch.equal(o, b)


def some(seed, sizes, dtypes, std=1e-2):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return [(torch.randn(n, device="cuda", generator=g) * std).to(d) for n, d in zip(sizes, dtypes)]


B, F = torch.bfloat16, torch.float32


@pytest.mark.parametrize("sizes,dtypes", [
    ([1], [B]), ([1], [F]), ([3, 0, 5], [B, F, F]), ([8192], [B]), ([8193, 8191, 2048, 7], [F, B, B, F]), ([100000, 1, 4097], [B, B, F]),
    ([5_000_011], [B]), ([3_000_001, 64], [F, B])])
@pytest.mark.parametrize("max_norm", [1e-3, 1e6])
def test_norm_and_clip(sizes, dtypes, max_norm):
    grads = some(sum(sizes), sizes, dtypes)
    check_clip(grads, max_norm, [torch.full_like(g, 9.0) for g in grads])
    check_clip(grads, max_norm)


def test_more_tensors_than_a_launch_takes():
    sizes = [(37 * i) % 301 for i in range(365)]
    check_clip(some(3, sizes, [B if i % 3 else F for i in range(365)]), 0.5)


@pytest.mark.parametrize("dtype", [B, F])
@pytest.mark.parametrize("skew_in,skew_out", [(0, 1), (1, 0), (1, 1), (3, 5)])
def test_every_alignment(dtype, skew_in, skew_out):
    base, out = some(5, [20000], [dtype])[0], torch.full((20000,), 9.0, dtype=dtype, device="cuda")
    n = 9001
    check_clip([base[skew_in:skew_in + n]], 0.1, [out[skew_out:skew_out + n]])
    assert bool((out[:skew_out] == 9.0).all()) and bool((out[skew_out + n:] == 9.0).all())


@pytest.mark.parametrize("dtype", [B, F])
@pytest.mark.parametrize("value,max_norm", [(1e30, 1.0), (3e38, 1e3), (1e-30, 1e-31)])
def test_squares_that_leave_binary32(dtype, value, max_norm):
    """Squares far above and far below what binary32 holds (the factor itself stays a normal number)."""
    check_clip([torch.full((1000,), value, dtype=dtype, device="cuda"), torch.full((7,), -value, dtype=dtype, device="cuda")], max_norm)


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_a_norm_that_is_not_finite_leaves_the_gradients(bad):
    grads = some(6, [5000, 30], [B, F])
    grads[1][3] = bad
    keep = [g.clone() for g in grads]
    outs = [torch.zeros_like(g) for g in grads]
    _, sumsq = norm_of(grads)
    norm = torch.zeros(1, device="cuda")
    fog.grad_clip(fog.make_grad_jobs(list(zip(grads, outs))), sumsq, 1e-3, norm)
    fog.grad_clip(fog.make_grad_jobs(grads), sumsq, 1e-3, norm)
    assert math.isnan(norm.item()) if math.isnan(bad) else norm.item() == math.inf
    for k, g, o in zip(keep, grads, outs):
        assert torch.equal(k.view(torch.uint8), g.view(torch.uint8)) and torch.equal(k.view(torch.uint8), o.view(torch.uint8))


def test_limits_of_zero_and_gradients_of_zero():
    check_clip(some(7, [300], [F]), 0.0)
    check_clip([torch.zeros(300, device="cuda", dtype=B)], 0.0)
    check_clip([torch.zeros(300, device="cuda", dtype=B)], 1.0)


def test_without_elements():
    jobs, sumsq = norm_of([torch.empty(0, device="cuda")])
    norm = torch.full((1,), 5.0, device="cuda")
    fog.grad_clip(jobs, sumsq, 1.0, norm)
    assert sumsq.item() == 0.0 and norm.item() == 0.0
    _, sumsq = norm_of([])
    assert sumsq.item() == 0.0


def test_the_sum_is_the_same_on_every_run():
    grads = some(8, [3_000_000, 77, 40_000], [B, F, F])
    assert len({norm_of(grads)[1].item() for _ in range(4)}) == 1


def test_sums_of_shards_add_up_to_the_whole_norm():
    """Two ranks' sums added before the clip, as their all-reduce would: both clip by the norm of the whole."""
    grads = some(9, [10000, 3000], [B, B])
    halves = [[g[:g.numel() // 2] for g in grads], [g[g.numel() // 2:].clone() for g in grads]]
    total = norm_of(halves[0])[1] + norm_of(halves[1])[1]
    norm = torch.zeros(1, device="cuda")
    want = math.sqrt(exact_sumsq(grads))
    fog.grad_clip(fog.make_grad_jobs(halves[1]), total, 1e-2, norm)
    assert abs(norm.item() - want) <= 2.0 ** -23 * want
    assert len(np.unique(norm.cpu().numpy())) == 1


def test_a_gradient_of_more_than_2_to_the_31_elements():
    n = (1 << 31) + 12345
    g = torch.full((n,), 2.0 ** -10, dtype=torch.bfloat16, device="cuda")
    g[-1] = 3.0
    _, sumsq = norm_of([g])
    assert sumsq.item() == (n - 1) * 2.0 ** -20 + 9.0          # every partial sum is a multiple of 2^-20 below 2^33: exact
    norm = torch.zeros(1, device="cuda")
    fog.grad_clip(fog.make_grad_jobs([g]), sumsq, math.sqrt(sumsq.item()) / 2, norm)
    # the factor is a half within a rounding or two: the products round to the exact halves
    assert bool((g[:-1] == 2.0 ** -11).all()) and g[-1].item() == 1.5
