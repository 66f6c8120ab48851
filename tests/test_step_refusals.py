"""Argument checks of the calls of a training step: host code, nothing is launched (no GPU needed)."""
import ctypes

import pytest
import torch

from paper_2505_20524_amd import fog

OK, NULL, SHAPE, ALIGN, UNSUPPORTED, WORKSPACE, HIP = range(7)
P = 1 << 20            # an address that is never followed: every call here is refused first
MB = 1 << 20


@pytest.fixture(scope="module")
def lib():
    return fog.load()


BF, F = fog.BF16, fog.F32
NAN, INF = float("nan"), float("inf")


def job(**change):
    a = dict(p=P, g=2 * P, master=3 * P, m=4 * P, v=5 * P, m_scale=6 * P, v_scale=7 * P, n=1000, p_type=BF, g_type=BF, weight_decay=0.1)
    a.update(change)
    return fog.AdamwJob(**a)


def adamw(lib, jobs=None, states=0, lr=1e-3, lr_dev=None, beta1=0.9, beta2=0.95, eps=1e-8, step=1, step_dev=None, seed=0, sumsq=None, max_norm=1.0, count=None):
    arr = (fog.AdamwJob * len(jobs))(*jobs) if jobs is not None else None
    return lib.fog_adamw(arr, len(jobs) if count is None else count, states, lr, lr_dev, beta1, beta2, eps, step, step_dev, seed, sumsq, max_norm, None)


@pytest.mark.parametrize("status,change", [
    (OK, dict(n=0)), (OK, dict(n=0, p=None, g=None, m=None, v=None)),
    (NULL, dict(p=None)), (NULL, dict(g=None)), (NULL, dict(m=None)), (NULL, dict(v=None)), (SHAPE, dict(n=-1)),
    (ALIGN, dict(p=P + 1)), (ALIGN, dict(g=P + 1)), (ALIGN, dict(master=P + 2)), (ALIGN, dict(m=P + 2)), (ALIGN, dict(v=P + 1)),
    (ALIGN, dict(p=P + 2, p_type=F, master=None)), (ALIGN, dict(g=P + 2, g_type=F)),
    (UNSUPPORTED, dict(p_type=2)), (UNSUPPORTED, dict(g_type=-1)), (UNSUPPORTED, dict(p_type=F)), (UNSUPPORTED, dict(weight_decay=NAN)),
    (UNSUPPORTED, dict(weight_decay=INF)), (UNSUPPORTED, dict(n=(1 << 36) + 1))])
def test_adamw_job(lib, status, change):
    assert adamw(lib, [job(**change)]) == status
    assert adamw(lib, [job(n=0), job(**change)]) == status


@pytest.mark.parametrize("status,change", [
    (NULL, dict(m_scale=None)), (NULL, dict(v_scale=None)), (UNSUPPORTED, dict(m_scale=P)), (UNSUPPORTED, dict(v_scale=6 * P))])
def test_adamw_job_of_fp8_states(lib, status, change):
    assert adamw(lib, [job(**change)], states=1) == status


@pytest.mark.parametrize("status,change", [
    (SHAPE, dict(count=-1)), (SHAPE, dict(step=0)), (NULL, dict(jobs=None, count=1)), (UNSUPPORTED, dict(jobs=None, count=(1 << 24) + 1)),
    (UNSUPPORTED, dict(states=2)), (UNSUPPORTED, dict(beta1=1.0)), (UNSUPPORTED, dict(beta1=-0.1)), (UNSUPPORTED, dict(beta2=1.0)), (UNSUPPORTED, dict(beta2=NAN)),
    (UNSUPPORTED, dict(states=1, beta2=0.999)), (UNSUPPORTED, dict(states=1, beta1=0.995)),
    (UNSUPPORTED, dict(eps=0.0)), (UNSUPPORTED, dict(eps=1e-39)), (UNSUPPORTED, dict(eps=INF)), (UNSUPPORTED, dict(lr=NAN)), (UNSUPPORTED, dict(lr=INF)),
    (UNSUPPORTED, dict(sumsq=P, max_norm=-1.0)), (UNSUPPORTED, dict(sumsq=P, max_norm=NAN)),
    (ALIGN, dict(lr_dev=P + 2)), (ALIGN, dict(step_dev=P + 4)), (ALIGN, dict(sumsq=P + 4))])
def test_adamw(lib, status, change):
    assert adamw(lib, **{**dict(jobs=[job()]), **change}) == status


@pytest.mark.parametrize("change", [
    dict(g=P), dict(master=P), dict(m=P + 1996), dict(v=4 * P), dict(master=4 * P - 4), dict(g=3 * P + 3998)])
def test_adamw_buffers_that_overlap(lib, change):
    assert adamw(lib, [job(**change)]) == UNSUPPORTED


def test_adamw_tensors_that_overlap(lib):
    far = dict(p=11 * P, g=12 * P, master=13 * P, m=14 * P, v=15 * P)
    assert adamw(lib, [job(), job()]) == UNSUPPORTED                                       # listed twice
    for name, at in far.items():
        assert adamw(lib, [job(), job(**{**far, name: 4 * P + 8})]) == UNSUPPORTED, name    # on the first one's m
    if not torch.cuda.is_available():
        assert adamw(lib, [job(), job(**{**far, "g": 2 * P})]) == HIP                       # one gradient read twice: taken, and no device to launch on


def test_the_binding_looks_at_types_and_sizes():
    n = 300
    good = dict(p=torch.zeros(n, dtype=torch.bfloat16), g=torch.zeros(n), m=torch.zeros(n), v=torch.zeros(n))
    assert fog.make_adamw_jobs([good]).states == fog.STATES_F32
    codes = dict(m=torch.zeros(n, dtype=torch.uint8), v=torch.zeros(n, dtype=torch.float8_e5m2), m_scale=torch.zeros(3, dtype=torch.uint8),
                 v_scale=torch.zeros(3, dtype=torch.uint8))
    assert fog.make_adamw_jobs([{**good, **codes}]).states == fog.STATES_FP8
    for bad in (dict(p=torch.zeros(n, dtype=torch.float16)), dict(g=torch.zeros(n - 1)), dict(m=torch.zeros(2 * n)[::2]), dict(v=torch.zeros(n, dtype=torch.float64)),
                dict(m=None), dict(master=torch.zeros(n, dtype=torch.bfloat16)), {**codes, "m_scale": None}, {**codes, "v_scale": torch.zeros(2, dtype=torch.uint8)},
                {**codes, "v": torch.zeros(n, dtype=torch.float8_e4m3fn)}):
        with pytest.raises(ValueError):
            fog.make_adamw_jobs([{**good, **bad}])
    with pytest.raises(ValueError):
        fog.make_adamw_jobs([good, {**good, **codes}])
    assert ctypes.sizeof(fog.AdamwJob) == 80


# ---------------------------------------------------------------------------------------------- rotary positions
def heads(p=P, batch=4096, token=256, head=128):
    return fog.Heads(p, batch, token, head)


def rope_job(heads_n=2, **change):
    a = dict(x=heads(), q=heads(P + MB), heads=heads_n, rotate=1, gain=1.0, fmt=0, scale=P, amax=P)
    a.update(change)
    return fog.RopeJob(**a)


def rope_grad_job(heads_n=2, **change):
    a = dict(dy=heads(), x=heads(P + MB), dx=heads(P + 2 * MB), q=heads(P + 3 * MB), heads=heads_n, rotate=1, gain=1.0, fmt=1, scale=P, amax=P)
    a.update(change)
    return fog.RopeGradJob(**a)


def rope(lib, jobs, grad=False, B=3, S=16, D=128, rot=128, layout=0, table=P, positions=16, pos=None, pos_bytes=0, offset=0, ws=P, ws_bytes=1 << 16, count=None):
    arr = ((fog.RopeGradJob if grad else fog.RopeJob) * len(jobs))(*jobs) if jobs is not None else None
    call = lib.fog_rope_grad if grad else lib.fog_rope_quantize
    return call(arr, len(jobs) if count is None else count, B, S, D, rot, layout, table, positions, pos, pos_bytes, offset, ws, ws_bytes, None)


CALLS = [
    (SHAPE, dict(count=-1)), (SHAPE, dict(count=9)), (NULL, dict(jobs=None, count=1)), (SHAPE, dict(B=-1)), (SHAPE, dict(S=-1)), (SHAPE, dict(D=-1, rot=-1)),
    (SHAPE, dict(rot=-2)), (SHAPE, dict(rot=130)), (SHAPE, dict(positions=-1)), (UNSUPPORTED, dict(rot=127)), (UNSUPPORTED, dict(D=1009)),
    (UNSUPPORTED, dict(layout=2)), (UNSUPPORTED, dict(layout=-1)), (UNSUPPORTED, dict(B=1 << 16, S=1 << 15)), (UNSUPPORTED, dict(pos=P, pos_bytes=2)),
    (UNSUPPORTED, dict(offset=-(1 << 63))), (ALIGN, dict(table=P + 2)), (ALIGN, dict(pos=P + 4, pos_bytes=8)), (ALIGN, dict(pos=P + 2, pos_bytes=4)),
    (NULL, dict(table=None)), (WORKSPACE, dict(ws=None)), (WORKSPACE, dict(ws_bytes=(1 << 16) - 1)), (ALIGN, dict(ws=P + 2))]


@pytest.mark.parametrize("status,change", CALLS)
@pytest.mark.parametrize("grad", [False, True])
def test_rope(lib, grad, status, change):
    make = rope_grad_job if grad else rope_job
    assert rope(lib, **{**dict(jobs=[make()]), **change}, grad=grad) == status


JOB = [
    (SHAPE, dict(heads_n=-1)), (UNSUPPORTED, dict(heads_n=(1 << 24) + 1)), (UNSUPPORTED, dict(fmt=2)), (UNSUPPORTED, dict(gain=-1.0)), (UNSUPPORTED, dict(gain=NAN)),
    (UNSUPPORTED, dict(gain=INF)), (NULL, dict(scale=None)), (ALIGN, dict(scale=P + 1)), (ALIGN, dict(amax=P + 2)), (NULL, dict(x=heads(None))),
    (ALIGN, dict(x=heads(P + MB + 1))), (SHAPE, dict(x=heads(P + MB, batch=-1))), (UNSUPPORTED, dict(x=heads(P + MB, token=1 << 60)))]


@pytest.mark.parametrize("status,change", JOB + [
    (NULL, dict(q=heads(None))), (SHAPE, dict(q=heads(P + MB, token=-1))),
    (SHAPE, dict(q=heads(P + MB, head=127))), (SHAPE, dict(q=heads(P + MB, head=0))), (SHAPE, dict(q=heads(P + MB, token=255))),      # vectors of q on each other
    (SHAPE, dict(q=heads(P + MB, batch=256))), (UNSUPPORTED, dict(q=heads(P)))])
def test_rope_job(lib, status, change):
    if "x" in change and change["x"].p == P + MB:
        change = {**change, "q": heads(P + 4 * MB)}
    assert rope(lib, [rope_job(**change)]) == status


@pytest.mark.parametrize("status,change", JOB + [
    (NULL, dict(dy=heads(None))), (NULL, dict(dx=heads(None), q=heads(None))), (ALIGN, dict(dx=heads(P + 2 * MB + 1))), (SHAPE, dict(dx=heads(P + 2 * MB, head=64))),
    (SHAPE, dict(q=heads(P + 3 * MB, head=64))), (UNSUPPORTED, dict(dx=heads(P))), (UNSUPPORTED, dict(dx=heads(P + MB))), (UNSUPPORTED, dict(q=heads(P + 2 * MB)))])
def test_rope_grad_job(lib, status, change):
    assert rope(lib, [rope_grad_job(**change)], grad=True) == status


def outputs(lib, a, b, **call):
    """Whether two jobs' codes may lie like this: HIP (there is no device to launch on) or UNSUPPORTED."""
    (pa, ha), (pb, hb) = a, b
    return rope(lib, [rope_job(ha, q=pa, amax=None), rope_job(hb, q=pb, amax=None)], **call)


@pytest.mark.skipif(torch.cuda.is_available(), reason="would be launched on addresses that are none")
def test_rope_outputs_that_lie_between_each_other(lib):
    Q = P + MB
    row = lambda first, n: (heads(Q + 128 * first, 16 * 1024, 1024, 128), n)  # noqa: E731      eight heads of 128 a token
    assert outputs(lib, row(0, 4), row(4, 4)) == HIP
    assert outputs(lib, row(4, 4), row(0, 4)) == HIP
    assert outputs(lib, row(0, 4), row(3, 4)) == UNSUPPORTED
    assert outputs(lib, row(0, 8), row(7, 1)) == UNSUPPORTED
    assert outputs(lib, row(0, 1), row(7, 1)) == HIP
    assert outputs(lib, row(0, 5), row(7, 1)) == HIP
    assert outputs(lib, row(0, 5), row(7, 2)) == UNSUPPORTED              # the second head lies in the next token's first
    assert outputs(lib, row(0, 4), row(4, 4), B=1) == HIP and outputs(lib, row(0, 4), row(4, 4), S=1) == HIP
    assert outputs(lib, row(0, 4), row(3, 4), B=1, S=1) == UNSUPPORTED
    kv = lambda i, n: (heads(Q + i * 16 * 1024, 2 * 16 * 1024, 128, 16 * 128), n)  # noqa: E731      [B, 2, 8 heads, 16 tokens, 128]
    assert outputs(lib, kv(0, 8), kv(1, 8)) == HIP and outputs(lib, kv(1, 8), kv(0, 8)) == HIP
    assert outputs(lib, kv(0, 8), kv(0, 8)) == UNSUPPORTED
    assert outputs(lib, kv(0, 8), row(0, 8)) == UNSUPPORTED               # other strides in the same range: not seen to lie apart
    assert outputs(lib, kv(0, 8), (heads(Q + MB, 4096, 256, 128), 2)) == HIP


def test_rope_outputs_on_the_table_or_the_positions(lib):
    end = P + 16 * 128 * 4                                                # of a table of 16 rows
    for at in (P, end - 1):
        assert rope(lib, [rope_job(q=heads(at), x=heads(P + 8 * MB))]) == UNSUPPORTED
        assert rope(lib, [rope_grad_job(dx=heads(at & ~1), dy=heads(P + 8 * MB))], grad=True) == UNSUPPORTED
    for pos_bytes in (4, 8):
        for at in (P + 2 * MB, P + 2 * MB + 48 * pos_bytes - 1):           # 3 x 16 positions
            assert rope(lib, [rope_job(q=heads(at))], pos=P + 2 * MB, pos_bytes=pos_bytes) == UNSUPPORTED
    assert rope(lib, [rope_job()], positions=1 << 60) == UNSUPPORTED
    if not torch.cuda.is_available():
        assert rope(lib, [rope_job(q=heads(end), x=heads(P + 8 * MB))]) == HIP
        assert rope(lib, [rope_job(q=heads(P + 2 * MB + 48 * 4))], pos=P + 2 * MB, pos_bytes=4) == HIP


def table(lib, first=0, positions=10, rot=64, t=P, **scaling):
    s = dict(base=10000.0, factor=2.0, low=1.0, high=4.0, original=4096.0, amplitude=1.0)
    s.update(scaling)
    return lib.fog_rope_table(ctypes.byref(fog.RopeScaling(**s)), first, positions, rot, t, None)


@pytest.mark.parametrize("status,change", [
    (OK, dict(positions=0)), (OK, dict(rot=0, t=None)), (NULL, dict(t=None)), (SHAPE, dict(positions=-1)), (SHAPE, dict(rot=-2)), (ALIGN, dict(t=P + 2)),
    (UNSUPPORTED, dict(rot=63)), (UNSUPPORTED, dict(positions=(1 << 31) + 1)), (UNSUPPORTED, dict(first=1 << 53)), (UNSUPPORTED, dict(base=0.0)), (UNSUPPORTED, dict(base=INF)),
    (UNSUPPORTED, dict(factor=0.0)), (UNSUPPORTED, dict(factor=NAN)), (UNSUPPORTED, dict(low=4.0)), (UNSUPPORTED, dict(high=NAN)), (UNSUPPORTED, dict(original=-1.0)),
    (UNSUPPORTED, dict(original=INF)), (UNSUPPORTED, dict(amplitude=NAN))])
def test_rope_table(lib, status, change):
    assert table(lib, **change) == status


def test_rope_bindings_look_at_types_and_shapes():
    x, q, s = torch.zeros((2, 3, 4, 8), dtype=torch.bfloat16), torch.zeros((2, 3, 4, 8), dtype=torch.uint8), torch.ones(1)
    good = dict(x=x, q=q, scale=s)
    assert fog.make_rope_jobs([good]).shape == (2, 3, 8)
    for bad in (dict(x=x.float()), dict(x=x[..., ::2]), dict(q=q[:, :2]), dict(q=q.view(torch.float8_e5m2)), dict(q=None), dict(scale=s.double()), dict(amax=s.half())):
        with pytest.raises((ValueError, AttributeError)):
            fog.make_rope_jobs([{**good, **bad}])
    with pytest.raises(ValueError):
        fog.make_rope_jobs([good, dict(x=x[:1], q=q[:1], scale=s)])
    with pytest.raises(ValueError):
        fog.rope_quantize(fog.make_rope_jobs([good]), None)          # to be turned, by no table
    assert ctypes.sizeof(fog.RopeJob) == 96 and ctypes.sizeof(fog.RopeGradJob) == 160


# ---------------------------------------------------------------------------------------------- gradients of post-norm and activations
def norm_grad(lib, dres=P, ld_dres=64, dbranch=P + MB, ld_dbranch=64, y=P + 2 * MB, ldy=64, rows=4, cols=64, gamma=P + 3 * MB, fmt=1, scale=P + 4 * MB, dstream=P + 5 * MB,
              ld_dstream=64, dy=P + 6 * MB, ld_dy=64, q=P + 7 * MB, ldq=64, amax=P, dgamma=P + 8 * MB, accumulate=0, ws=P, ws_bytes=1 << 30):
    return lib.fog_postnorm_residual_grad(dres, ld_dres, dbranch, ld_dbranch, y, ldy, rows, cols, gamma, fmt, scale, dstream, ld_dstream, dy, ld_dy, q, ldq, amax,
                                          dgamma, accumulate, ws, ws_bytes, None)


NORM = [
    (OK, dict(rows=0, amax=None, dgamma=None)), (OK, dict(rows=0, amax=None, accumulate=1)), (OK, dict(cols=0, amax=None)),
    (NULL, dict(dres=None)), (NULL, dict(y=None)), (NULL, dict(gamma=None)), (NULL, dict(scale=None)), (SHAPE, dict(rows=-1)), (SHAPE, dict(cols=-1)),
    (SHAPE, dict(ld_dres=63)), (SHAPE, dict(ld_dbranch=63)), (SHAPE, dict(ldy=63)), (SHAPE, dict(ld_dstream=63)), (SHAPE, dict(ld_dy=63)), (SHAPE, dict(ldq=63)),
    (ALIGN, dict(dres=P + 1)), (ALIGN, dict(dbranch=P + MB + 1)), (ALIGN, dict(y=P + 2 * MB + 1)), (ALIGN, dict(dstream=P + 5 * MB + 1)), (ALIGN, dict(dy=P + 6 * MB + 1)),
    (ALIGN, dict(gamma=P + 3 * MB + 2)), (ALIGN, dict(dgamma=P + 8 * MB + 2)), (ALIGN, dict(amax=P + 1)), (ALIGN, dict(scale=P + 1)), (ALIGN, dict(ws=P + 2)),
    (WORKSPACE, dict(ws=None)), (WORKSPACE, dict(ws_bytes=64 * 4 + 3)), (UNSUPPORTED, dict(fmt=2)), (UNSUPPORTED, dict(cols=32769)),
    (UNSUPPORTED, dict(ldy=1 << 60)),
    # results on inputs and on each other
    (UNSUPPORTED, dict(dstream=P + 2)), (UNSUPPORTED, dict(dy=P + 5 * MB)), (UNSUPPORTED, dict(q=P + 6 * MB + 100)), (UNSUPPORTED, dict(dgamma=P + 7 * MB)),
    (UNSUPPORTED, dict(dstream=P, ld_dstream=80)), (UNSUPPORTED, dict(dy=P, dstream=P)), (UNSUPPORTED, dict(q=P)), (UNSUPPORTED, dict(dy=P + 3 * MB - 4)),
    (UNSUPPORTED, dict(dstream=P + 64, ld_dres=96, ld_dstream=96))]


@pytest.mark.parametrize("status,change", NORM)
def test_postnorm_grad(lib, status, change):
    assert norm_grad(lib, **change) == status


@pytest.mark.skipif(torch.cuda.is_available(), reason="would be launched on addresses that are none")
@pytest.mark.parametrize("change", [
    {}, dict(dstream=P), dict(dstream=P + MB), dict(dy=P + 2 * MB), dict(dy=P), dict(dbranch=P), dict(dbranch=None, dstream=None), dict(q=None, scale=None),
    dict(amax=None, dgamma=None, ws=None), dict(dstream=P + 2 * 64, ld_dres=128, ld_dstream=128)])      # the last: the columns beside
def test_postnorm_grad_takes(lib, change):
    assert norm_grad(lib, **change) == HIP


def test_postnorm_grad_workspace(lib):
    size = lib.fog_postnorm_residual_grad_workspace
    assert size(0, 64) == 0 and size(4, 0) == 0 and size(4, 32769) == 0 and size(-1, -1) == 0
    assert size(1, 64) == 64 * 4 + 4 and size(8, 64) == size(1, 64) and size(9, 64) == 2 * size(1, 64) and size(1 << 40, 64) == 512 * size(1, 64)
    assert size(1 << 40, 4096) == 512 * (4 * 4096 + 4) and size(1 << 40, 16384) == 512 * (4 * 16384 + 4) and size(1 << 40, 32768) == 512 * (4 * 32768 + 4)


def act_grad(lib, which, x=P, ldx=64, dy=P + MB, ld_dy=64, rows=4, cols=64, alpha=(0.8, 0.6), fmt=1, scale=P + 2 * MB, dx=P + 3 * MB, ld_dx=64, q=P + 4 * MB, ldq=64,
             amax=P, dalpha=P, accumulate=0, ws=P, ws_bytes=1 << 20):
    own = () if which == "gelu" else (dalpha, accumulate)
    params = {"xielu": alpha, "tanh": alpha[:1], "gelu": ()}[which]
    return getattr(lib, "fog_%s_grad" % which)(x, ldx, dy, ld_dy, rows, cols, *params, fmt, scale, dx, ld_dx, q, ldq, amax, *own, ws, ws_bytes, None)


@pytest.mark.parametrize("which", ["xielu", "gelu", "tanh"])
@pytest.mark.parametrize("status,change", [
    (OK, dict(rows=0, amax=None, dalpha=None)), (OK, dict(cols=0, amax=None, accumulate=1)),
    (NULL, dict(x=None)), (NULL, dict(dy=None)), (NULL, dict(scale=None)), (SHAPE, dict(rows=-1)), (SHAPE, dict(cols=-1)), (SHAPE, dict(ldx=63)), (SHAPE, dict(ld_dy=63)),
    (SHAPE, dict(ld_dx=63)), (SHAPE, dict(ldq=63)), (ALIGN, dict(x=P + 1)), (ALIGN, dict(dy=P + MB + 1)), (ALIGN, dict(dx=P + 3 * MB + 1)), (ALIGN, dict(amax=P + 2)),
    (ALIGN, dict(scale=P + 2)), (ALIGN, dict(ws=P + 4)), (WORKSPACE, dict(ws=None)), (WORKSPACE, dict(ws_bytes=2048 * 20 - 1)), (UNSUPPORTED, dict(fmt=3)),
    (UNSUPPORTED, dict(rows=1 << 40, cols=1 << 20, ldx=1 << 20, ld_dy=1 << 20, ld_dx=1 << 20, ldq=1 << 20)),
    (UNSUPPORTED, dict(dx=P + 2)), (UNSUPPORTED, dict(q=P)), (UNSUPPORTED, dict(q=P + 3 * MB + 4)), (UNSUPPORTED, dict(dx=P, ld_dx=80))])
def test_act_grad(lib, which, status, change):
    assert act_grad(lib, which, **change) == status


@pytest.mark.parametrize("which,alpha", [("xielu", (-0.1, 0.0)), ("xielu", (0.0, -1.0)), ("xielu", (NAN, 0.0)), ("xielu", (0.0, INF)), ("tanh", (NAN,)), ("tanh", (INF,))])
def test_act_grad_parameters(lib, which, alpha):
    assert act_grad(lib, which, alpha=alpha) == UNSUPPORTED


@pytest.mark.skipif(torch.cuda.is_available(), reason="would be launched on addresses that are none")
@pytest.mark.parametrize("which", ["xielu", "gelu", "tanh"])
def test_act_grad_takes(lib, which):
    for change in ({}, dict(dx=P), dict(dx=P + MB), dict(dx=None), dict(q=None, scale=None), dict(amax=None, dalpha=None, ws=None), dict(x=P + MB)):
        assert act_grad(lib, which, **change) == HIP
