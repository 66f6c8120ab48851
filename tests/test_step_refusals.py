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
    (UNSUPPORTED, dict(weight_decay=INF)), (UNSUPPORTED, dict(n=(1 << 37) + 1))])
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
