"""GPU parity at the largest table that the embedding's gradient takes: ids whose sort keys fill their 32 bits, beside ids just outside."""
import numpy as np
import pytest
import torch

from oracle import bf16
from paper_2505_20524_amd import fog
from parity import dev

pytestmark = pytest.mark.gpu

V = 4194302


@pytest.mark.parametrize("T", [50, 2048, 2049, 5000])          # ordered by ranking up to 2048 tokens, by tiles and a merge above
@pytest.mark.parametrize("accumulate", [False, True])
def test_the_last_ids_of_the_largest_table(T, accumulate):
    rng = np.random.default_rng(T)
    H = 8
    ids = np.array([V - 1, V - 2, 0, 1, V // 2, V, V + 1, V + 2, (1 << 22), (1 << 31) - 1, -1, -(1 << 31)])
    tokens = rng.choice(ids, T)
    # whole numbers: sums of up to 5000 of them are exact in binary32 in any order
    dx = rng.integers(-8, 9, (T, H)).astype(np.float64)
    dE = torch.full((V, H), 3.0, device="cuda")
    ws = torch.full((fog.embed_grad_workspace(T, V, H),), 0xFF, dtype=torch.uint8, device="cuda")
    fog.embed_grad(dev(tokens), dev(bf16.f64_to_bits_rne(dx)), 2.0, dE, ws, accumulate=accumulate)
    start = 3.0 if accumulate else 0.0
    for v in (V - 1, V - 2, 0, 1, V // 2):
        assert np.array_equal(dE[v].double().cpu().numpy(), start + 2.0 * dx[tokens == v].sum(0)), v
        dE[v] = start
    assert bool((dE == start).all())
    x = torch.full((T, H), 5.0, dtype=torch.bfloat16, device="cuda")
    table = torch.zeros((V, H), dtype=torch.bfloat16, device="cuda")
    table[V - 2], table[V - 1], table[0] = 1.0, 2.0, 7.0
    fog.embed_quantize(dev(tokens), table, 1.0, fog.E4M3, None, x)
    want = np.select([tokens == V - 2, tokens == V - 1, tokens == 0], [1.0, 2.0, 7.0], 0.0)
    assert np.array_equal(x.double().cpu().numpy(), np.repeat(want[:, None], H, 1))
