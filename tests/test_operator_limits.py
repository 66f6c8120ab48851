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


def embed_grad(lib, count, vocab, cols, ld_dE=None, type=1, accumulate=0, dE=None):
    return lib.fog_embed_grad(P, 8, count, P, cols, vocab, cols, 1.0, type, dE, ld_dE or cols, accumulate, P, 0, None)


# ceil(count / 64) * ceil(cols / 512) against 2^22: columns count in whole pieces of 512, tokens in whole 64
@pytest.mark.parametrize("count,cols,inside", [
    (1 << 28, 512, True), ((1 << 28) + 1, 512, False), (1 << 28, 1, True), ((1 << 28) + 1, 1, False), (1 << 28, 513, False), (1 << 27, 513, True),
    ((1 << 27) + 1, 513, False), (200_000_000, 600, False), (64, (1 << 31) - 1, True), (65, (1 << 31) - 1, False), (1, (1 << 31) - 1, True)])
@pytest.mark.parametrize("accumulate", [0, 1])
def test_tokens_and_columns_of_an_embeddings_gradient(lib, count, cols, inside, accumulate):
    """The query has room for what the call takes and none for what it refuses."""
    assert embed_grad(lib, count, 10, cols, accumulate=accumulate) == (NULL if inside else UNSUPPORTED)
    assert embed_grad(lib, count, 10, cols, accumulate=accumulate, dE=P) == (WORKSPACE if inside else UNSUPPORTED)
    assert (lib.fog_embed_grad_workspace(count, 10, cols) > 0) == inside


@pytest.mark.parametrize("vocab,cols,type,inside", [
    (4194302, 1 << 20, 1, True), (4194302, (1 << 20) + 1, 1, False), (4194302, 1 << 21, 0, True), (4194302, (1 << 21) + 1, 0, False),
    (2048, (1 << 31) - 1, 1, False), (2047, (1 << 31) - 1, 1, True)])
def test_rows_of_a_strided_gradient_that_is_overwritten(lib, vocab, cols, type, inside):
    assert embed_grad(lib, 0, vocab, cols, ld_dE=cols + 1, type=type) == (NULL if inside else UNSUPPORTED)
    assert embed_grad(lib, 0, vocab, cols, type=type) == NULL                                     # rows that lie end to end
    assert embed_grad(lib, 1, vocab, cols, ld_dE=cols + 1, type=type, accumulate=1) == NULL       # nothing is cleared


def test_a_table_without_rows_has_no_limit(lib):
    assert embed_grad(lib, 1 << 30, 0, 1 << 20) == OK


def test_number_of_gradients(lib):
    """What a call sums is counted in 32 bits: up to 2^24 tensors, 4096 sums for each 120 of them."""
    most = 1 << 24
    for count, inside in ((most, True), (most + 1, False), ((1 << 31) - 1, False)):
        # nothing of the jobs is looked at before their number
        assert lib.fog_grad_sumsq(None, count, P, None, 0, None) == (NULL if inside else UNSUPPORTED)
        assert lib.fog_grad_clip(None, count, P, 1.0, None, None) == (NULL if inside else UNSUPPORTED)
        assert lib.fog_grad_sumsq_workspace(count) == (-(-count // 120) * 4096 * 8 if inside else 0)
