"""When the gradient of an embedding is one launch, which needs no workspace: neither with many tokens a
row of the table, nor with so many columns that a part of them has fewer than four blocks."""
import pytest


@pytest.fixture(scope="module")
def native():
    from paper_2505_00793_gb300 import build, native
    build.build()
    return native


@pytest.mark.parametrize("n,vocab,dim,dual,one", [
    (6144, 8192, 512, False, True), (6145, 8192, 512, False, False),
    (0, 1, 1, False, True), (1024, 1, 128, False, True), (1025, 1, 128, False, False), (6144, 1, 16, True, False),
    (2048, 2, 24, True, True), (2049, 2, 24, True, False), (6144, 6, 128, False, True), (6144, 5, 128, False, False),
    (500, 300, 76 * 128, False, True), (500, 300, 76 * 128 + 1, False, False),
    (500, 300, 38 * 128, True, True), (500, 300, 38 * 128 + 1, True, False), (500, 300, 2 ** 20, True, False),
    (40, 304 * 8192, 3, False, True), (40, 304 * 8192 + 1, 3, False, False)])
def test_one_launch(native, n, vocab, dim, dual, one):
    assert (native.mf_embed_work_bytes(n, vocab, dim, dual) == 16) == one
