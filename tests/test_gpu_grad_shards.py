"""GPU parity: gradients that are spread over ranks.  Every rank sums its own, the sums are added as the ranks' all-reduce would, and every rank clips
its own by the norm of the whole."""
import math

import pytest
import torch

from paper_2505_20524_amd import fog

pytestmark = pytest.mark.gpu

B, F = torch.bfloat16, torch.float32


def shards(sizes, stds, dtypes):
    """One list of gradients for each rank, with magnitudes of its own."""
    g = torch.Generator(device="cuda")
    g.manual_seed(sum(sum(s) for s in sizes))
    return [[(torch.randn(n, device="cuda", generator=g) * std).to(d) for n, d in zip(s, dtypes)] for s, std in zip(sizes, stds)]


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("sizes,stds,dtypes", [
    ([(10000, 3000), (10000, 3000)], (1e-2, 1e-2), (B, B)), ([(8193, 1, 77), (5, 100000, 0)], (1e-2, 3e-3), (F, B, B)),
    ([(9001,), (4000,), (20000,)], (1.0, 1e-3, 1e-2), (F,))])
def test_every_rank_clips_by_the_norm_of_the_whole(sizes, stds, dtypes, in_place):
    ranks = shards(sizes, stds, dtypes)
    sums = []
    for grads in ranks:
        s = torch.zeros(1, dtype=torch.float64, device="cuda")
        fog.grad_sumsq(fog.make_grad_jobs(grads), s, torch.empty(fog.grad_sumsq_workspace(len(grads)), dtype=torch.uint8, device="cuda"))
        sums.append(s)
    whole = torch.stack(sums).sum(0)
    own = [math.sqrt(math.fsum(float((g.double() ** 2).sum()) for g in grads)) for grads in ranks]
    norm = math.sqrt(math.fsum(r * r for r in own))
    max_norm = norm / 3
    n = sum(g.numel() for grads in ranks for g in grads)
    for grads, mine in zip(ranks, own):
        before = [g.clone() for g in grads]
        outs = grads if in_place else [torch.full_like(g, 9.0) for g in grads]
        told = torch.zeros(1, device="cuda")
        fog.grad_clip(fog.make_grad_jobs(grads if in_place else list(zip(grads, outs))), whole, max_norm, told)
        # binary64 sums of n squares in any order on both sides, one rounding to binary32
        assert abs(told.item() - norm) <= (2.0 ** -24 + (n + 8) * 2.0 ** -53) * norm
        for b, g, o in zip(before, grads, outs):
            want = b.double() * (max_norm / norm)
            # the limit and the factor as binary32, the product as binary32 (for bfloat16 within the one per cent) and as the type; results
            # below the normal range by a step of the subnormals
            rel = (2 * 2.0 ** -24 + (n + 8) * 2.0 ** -53 + torch.finfo(b.dtype).eps / 2) * 1.01
            assert bool(((o.double() - want).abs() <= rel * want.abs() + (2.0 ** -133 if b.dtype == B else 2.0 ** -149)).all())
            assert in_place or torch.equal(g, b)
            # a factor made of the rank's own norm would be seen
            assert abs(norm / mine - 1.0) > 4 * rel
