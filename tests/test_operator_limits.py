"""Limits of sizes: the largest that a call takes and the first that it refuses.  Host code, nothing is launched (no GPU needed): what is inside
the limit is told from what is not by an error that is looked for later, a missing pointer."""
import pytest

from paper_2505_20524_amd import fog

OK, NULL, SHAPE, ALIGN, UNSUPPORTED, WORKSPACE = range(6)
P = 1 << 20            # an address that is never followed: every call here is refused first


@pytest.fixture(scope="module")
def lib():
    return fog.load()


@pytest.mark.parametrize("cols,status", [((1 << 32) - 8, NULL), ((1 << 32) - 7, UNSUPPORTED), (1 << 32, UNSUPPORTED), ((1 << 32) + 8, UNSUPPORTED),
                                         (1 << 33, UNSUPPORTED), ((1 << 33) + 8, UNSUPPORTED)])
@pytest.mark.parametrize("count", [1, 3])
def test_columns_of_an_embedding(lib, cols, status, count):
    """Columns are counted in 32 bits, eight at a time."""
    for x in (None,) if status == NULL else (None, P):
        assert lib.fog_embed_quantize(P, 8, count, P, 10, cols, cols, 1.0, 0, None, x, cols, None, 0, None, None) == status
