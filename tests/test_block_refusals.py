"""Argument checks of the block-scaled calls, the embedding and the gradient norm: host code, nothing is launched (no GPU needed)."""
import ctypes

import pytest
import torch

from paper_2505_20524_amd import fog

OK, NULL, SHAPE, ALIGN, UNSUPPORTED, WORKSPACE = range(6)
P = 1 << 20            # an address that is never followed: every call here is refused first


@pytest.fixture(scope="module")
def lib():
    return fog.load()


def cast(lib, x=P, rows=4, cols=256, ldx=256, fmt=0, margin=0, q_row=P, ldq_row=256, s_row=P, lds_row=4, q_col=P, ldq_col=256, s_col=P, lds_col=256):
    return lib.fog_quantize_block(x, rows, cols, ldx, fmt, margin, q_row, ldq_row, s_row, lds_row, q_col, ldq_col, s_col, lds_col, None)


@pytest.mark.parametrize("status,change", [
    (OK, dict(rows=0)), (OK, dict(cols=0, x=None)),
    (NULL, dict(x=None)), (NULL, dict(q_row=None)), (NULL, dict(s_row=None)), (NULL, dict(q_col=None)), (NULL, dict(s_col=None)),
    (NULL, dict(q_row=None, s_row=None, q_col=None, s_col=None)),
    (SHAPE, dict(rows=-1)), (SHAPE, dict(cols=-1)), (SHAPE, dict(ldx=255)), (SHAPE, dict(ldq_row=255)), (SHAPE, dict(ldq_col=255)),
    (SHAPE, dict(lds_row=3)), (SHAPE, dict(lds_col=255)), (SHAPE, dict(margin=65)), (SHAPE, dict(margin=-65)),
    (ALIGN, dict(x=P + 1)), (UNSUPPORTED, dict(fmt=2))])
def test_quantize_block(lib, status, change):
    assert cast(lib, **change) == status


@pytest.mark.parametrize("status,change", [
    (OK, dict(rows=0)), (NULL, dict(x=None)), (NULL, dict(q=None)), (NULL, dict(s=None)), (SHAPE, dict(cols=-1)), (SHAPE, dict(ldx=299)),
    (SHAPE, dict(ldq=299)), (SHAPE, dict(lds=2)), (SHAPE, dict(margin=100)), (ALIGN, dict(x=P + 1)), (UNSUPPORTED, dict(fmt=-1))])
def test_quantize_tile(lib, status, change):
    a = dict(x=P, rows=4, cols=300, ldx=300, fmt=0, margin=0, q=P, ldq=300, s=P, lds=3)
    a.update(change)
    assert lib.fog_quantize_tile(a["x"], a["rows"], a["cols"], a["ldx"], a["fmt"], a["margin"], a["q"], a["ldq"], a["s"], a["lds"], None) == status


def gemm(lib, layout=0, M=256, N=512, K=384, A=P, fa=0, lda=512, ba=0, sA=P, ldsA=512, B=P, fb=0, ldb=512, bb=1, sB=P, ldsB=4, C=P, ldc=512):
    return lib.fog_fp8_gemm_block(layout, M, N, K, A, fa, lda, ba, sA, ldsA, B, fb, ldb, bb, sB, ldsB, C, ldc, None, 0, None)


@pytest.mark.parametrize("status,change", [
    (OK, dict(M=0)), (OK, dict(N=0)),
    (NULL, dict(C=None)), (NULL, dict(A=None)), (NULL, dict(B=None)), (NULL, dict(sA=None)), (NULL, dict(sB=None)),
    (SHAPE, dict(K=-1)), (SHAPE, dict(lda=368)), (SHAPE, dict(ldb=368)), (SHAPE, dict(ldc=511)),
    (SHAPE, dict(ldsA=255)),                                    # VECTOR: a byte for each of the 256 rows
    (SHAPE, dict(ldsB=2)),                                      # TILE of B [512, 384] as stored: three blocks of columns
    (SHAPE, dict(layout=1, ldsB=3)),                            # TILE of B [384, 512]: four
    (SHAPE, dict(layout=2, ba=1, ldsA=1)),                      # TILE of A [384, 256]: two
    (ALIGN, dict(A=P + 8)), (ALIGN, dict(lda=488)), (ALIGN, dict(C=P + 1)),
    (UNSUPPORTED, dict(K=392)), (UNSUPPORTED, dict(layout=3)), (UNSUPPORTED, dict(fa=2)), (UNSUPPORTED, dict(ba=2)), (UNSUPPORTED, dict(bb=-1)),
    (UNSUPPORTED, dict(ldsA=1 << 31))])
def test_gemm_block(lib, status, change):
    assert gemm(lib, **change) == status


@pytest.mark.parametrize("status,change", [
    (OK, dict(count=0)), (OK, dict(cols=0)), (NULL, dict(tokens=None)), (NULL, dict(table=None)), (NULL, dict(x=None)), (NULL, dict(scale=None)),
    (SHAPE, dict(count=-1)), (SHAPE, dict(vocab=-1)), (SHAPE, dict(ld_table=63)), (SHAPE, dict(ldx=63)), (SHAPE, dict(ldq=63)),
    (ALIGN, dict(tokens=P + 4)), (ALIGN, dict(table=P + 1)), (ALIGN, dict(x=P + 1)),
    (UNSUPPORTED, dict(bytes=2)), (UNSUPPORTED, dict(fmt=3)), (UNSUPPORTED, dict(factor=float("nan"))), (UNSUPPORTED, dict(factor=float("inf")))])
def test_embed_quantize(lib, status, change):
    a = dict(tokens=P, bytes=8, count=5, table=P, vocab=10, cols=64, ld_table=64, factor=1.0, fmt=0, scale=P, x=P, ldx=64, q=P, ldq=64)
    a.update(change)
    assert lib.fog_embed_quantize(a["tokens"], a["bytes"], a["count"], a["table"], a["vocab"], a["cols"], a["ld_table"], a["factor"], a["fmt"], a["scale"],
                                  a["x"], a["ldx"], a["q"], a["ldq"], None, None) == status


@pytest.mark.parametrize("status,change", [
    (OK, dict(vocab=0)), (OK, dict(cols=0)), (OK, dict(count=0, accumulate=1)),
    (NULL, dict(tokens=None)), (NULL, dict(dx=None)), (NULL, dict(dE=None)),
    (SHAPE, dict(count=-1)), (SHAPE, dict(ld_dx=63)), (SHAPE, dict(ld_dE=63)),
    (ALIGN, dict(tokens=P + 2)), (ALIGN, dict(dx=P + 1)), (ALIGN, dict(dE=P + 2)), (ALIGN, dict(ws=P + 8)),
    (WORKSPACE, dict(ws=None)), (WORKSPACE, dict(short=1)),
    (UNSUPPORTED, dict(bytes=1)), (UNSUPPORTED, dict(type=2)), (UNSUPPORTED, dict(factor=float("inf"))), (UNSUPPORTED, dict(vocab=4194303)),
    (UNSUPPORTED, dict(count=1 << 31))])
def test_embed_grad(lib, status, change):
    a = dict(tokens=P, bytes=4, count=1500, dx=P, ld_dx=64, vocab=10, cols=64, factor=1.0, type=1, dE=P, ld_dE=64, accumulate=0, ws=P, short=0)
    a.update(change)
    need = lib.fog_embed_grad_workspace(a["count"], a["vocab"], a["cols"]) - a["short"]
    assert lib.fog_embed_grad(a["tokens"], a["bytes"], a["count"], a["dx"], a["ld_dx"], a["vocab"], a["cols"], a["factor"], a["type"], a["dE"], a["ld_dE"],
                              a["accumulate"], a["ws"], max(need, 0), None) == status


def jobs(**change):
    a = dict(g=P, out=P, n=100, type=0)
    a.update(change)
    return (fog.GradJob * 1)(fog.GradJob(a["g"], a["out"], a["n"], a["type"]))


@pytest.mark.parametrize("sumsq,clip,change", [
    (NULL, NULL, dict(g=None)), (WORKSPACE, NULL, dict(out=None)), (SHAPE, SHAPE, dict(n=-1)), (ALIGN, ALIGN, dict(g=P + 1)),
    (ALIGN, ALIGN, dict(g=P + 2, type=1)), (WORKSPACE, ALIGN, dict(out=P + 1)), (UNSUPPORTED, UNSUPPORTED, dict(type=5)),
    (UNSUPPORTED, UNSUPPORTED, dict(n=(1 << 37) + 1))])
def test_grad_jobs(lib, sumsq, clip, change):
    j = jobs(**change)
    assert lib.fog_grad_sumsq(j, 1, P, None, 0, None) == sumsq
    assert lib.fog_grad_clip(j, 1, P, 1.0, None, None) == clip


def test_grad_calls(lib):
    j = jobs()
    assert lib.fog_grad_sumsq(j, -1, P, P, 1 << 20, None) == SHAPE
    assert lib.fog_grad_sumsq(None, 1, P, P, 1 << 20, None) == NULL
    assert lib.fog_grad_sumsq(j, 1, None, P, 1 << 20, None) == NULL
    assert lib.fog_grad_sumsq(j, 1, P + 4, P, 1 << 20, None) == ALIGN
    assert lib.fog_grad_sumsq(j, 1, P, P, lib.fog_grad_sumsq_workspace(1) - 1, None) == WORKSPACE
    assert lib.fog_grad_sumsq(j, 1, P, P + 4, 1 << 20, None) == ALIGN
    assert lib.fog_grad_clip(j, 1, None, 1.0, None, None) == NULL
    for bad in (-1.0, float("nan")):
        assert lib.fog_grad_clip(j, 1, P, bad, None, None) == UNSUPPORTED


def test_workspace_queries(lib):
    assert lib.fog_grad_sumsq_workspace(0) == 0
    assert lib.fog_grad_sumsq_workspace(121) == 2 * lib.fog_grad_sumsq_workspace(120) == 2 * lib.fog_grad_sumsq_workspace(1)
    assert lib.fog_embed_grad_workspace(0, 10, 64) == 0
    assert lib.fog_embed_grad_workspace(1, 10, 64) >= 2 * 4 + 2 * 256
    assert lib.fog_fp8_gemm_block_workspace(0, 4096, 8192, 2048) == lib.fog_fp8_gemm_workspace(0, 4096, 8192, 2048)


def test_the_binding_refuses_tensors_that_the_call_would_misread():
    x, q, s = torch.zeros((4, 256), dtype=torch.bfloat16), torch.zeros((4, 256), dtype=torch.uint8), torch.zeros((2, 4), dtype=torch.uint8)
    for bad in (dict(x=x.t()), dict(x=x.float()), dict(q_row=q[:3]), dict(q_row=q.t()), dict(s_row=s.t())):
        a = dict(x=x, q_row=q, s_row=s)
        a.update(bad)
        with pytest.raises(ValueError):
            fog.quantize_block(a["x"], fog.E4M3, q_row=a["q_row"], s_row=a["s_row"])
    with pytest.raises(ValueError):
        fog.fp8_gemm_block(fog.NT, 4, 4, 256, q, fog.E4M3, fog.VECTOR, s, q, fog.E4M3, fog.TILE, s[:, :1], torch.zeros((4, 4), dtype=torch.bfloat16))
    with pytest.raises(ValueError):
        fog.embed_quantize(torch.zeros(3), x, 1.0, fog.E4M3, None, x)
    with pytest.raises(ValueError):
        fog.make_grad_jobs([(x, x.float())])
    with pytest.raises(ValueError):
        fog.make_grad_jobs([x.t()])
    with pytest.raises(ValueError):
        fog.grad_sumsq(fog.make_grad_jobs([x]), torch.zeros(1), s)
    with pytest.raises(ValueError):
        fog.fp8_gemm_block(fog.NT, 4, 4, 256, q, fog.E4M3, fog.VECTOR, s, q, fog.E4M3, fog.TILE, torch.zeros((1, 2), dtype=torch.uint8),
                           torch.zeros((4, 4), dtype=torch.bfloat16), workspace=torch.zeros(1, dtype=torch.uint8).expand(1 << 20))
    assert ctypes.sizeof(fog.GradJob) == 32
