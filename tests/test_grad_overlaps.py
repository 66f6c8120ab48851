"""Gradients and clipped gradients that share memory: host code, nothing is launched (no GPU needed).  What the check lets through is told by a
HIP error (no GPU) or, where there is one, tested on real tensors in test_gpu_grad.py."""
import random

import pytest
import torch

from paper_2505_20524_amd import fog

HIP, UNSUPPORTED = 6, 4
P = 1 << 20


def clip(items):
    """items: (g, out, n, type) -> status of a clip of them."""
    jobs = (fog.GradJob * len(items))(*[fog.GradJob(*i) for i in items])
    return fog.load().fog_grad_clip(jobs, len(items), P, 1.0, None, None)


BF, F = fog.BF16, fog.F32
REFUSED = [
    [(P, P, 100, BF), (P, P, 100, BF)],                                     # listed twice
    [(P, P, 100, BF), (P + 4096, P + 4096, 8, BF), (P, P, 100, BF)],
    [(P, P, 100, BF), (P + 198, P + 198, 1, BF)],                           # the last element of another
    [(P, P, 100, F), (P + 396, P + 396, 1, F)],
    [(P, P + 2, 100, BF)],                                                  # a result that lies across its own gradient
    [(P + 198, P, 100, BF)],
    [(P, P + 4096, 100, BF), (P + 4096, P + 8192, 100, BF)],                # a result on another's gradient
    [(P, P + 4096, 100, BF), (P + 512, P + 4096 + 198, 100, BF)],           # results on each other
    [(P, P + 4096, 100, BF), (P + 4096 + 198, P + 4096 + 198, 1, BF)],
    [(P, P, 1 << 20, F), (P + 64, P + 64, 1, BF), (P + (3 << 20), P + (3 << 20), 1, BF)],      # inside a large one, another behind the small
]
TAKEN = [
    [(P, P, 100, BF), (P + 200, P + 200, 100, BF)],                         # end to end
    [(P + 400, P + 400, 100, F), (P, P, 100, F)],
    [(P, P + 200, 100, BF)],
    [(P, P + 4096, 100, BF), (P, P + 8192, 100, BF)],                       # one gradient read twice
    [(P, P + 4096, 100, BF), (P + 100, P + 8192, 100, BF)],
    [(P, P, 100, BF), (P, P, 0, BF), (P + 50, None, 0, F)],                 # no elements
]


@pytest.mark.parametrize("items", REFUSED)
def test_what_shares_memory_with_a_result_is_refused(items):
    for order in (items, items[::-1]):
        assert clip(order) == UNSUPPORTED


@pytest.mark.skipif(torch.cuda.is_available(), reason="would be launched on addresses that are none")
@pytest.mark.parametrize("items", TAKEN)
def test_what_lies_apart_is_taken(items):
    for order in (items, items[::-1]):
        assert clip(order) == HIP


@pytest.mark.skipif(torch.cuda.is_available(), reason="would be launched on addresses that are none")
def test_many_gradients():
    """More than the check keeps on the stack, in any order; one of them twice."""
    items = [(P + 8192 * i, P + 8192 * i, 4096, BF) for i in range(700)]
    random.Random(1).shuffle(items)
    assert clip(items) == HIP
    assert clip(items + [items[350]]) == UNSUPPORTED
    x, y, n, t = items[350]
    assert clip(items + [(x + 8190, y + 8190, 1, t)]) == UNSUPPORTED
