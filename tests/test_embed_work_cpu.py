"""The workspace of an embedding's gradient is asked for with the args of the call, whichever of its
tangents they hold."""
import ctypes as C

import pytest


@pytest.fixture(scope="module")
def native():
    from paper_2505_00793_gb300 import build, native
    build.build()
    return native


@pytest.mark.parametrize("n,vocab,dim", [(0, 200000, 1024), (0, 70, 20), (9000, 1000, 64), (40, 304 * 8192 + 1, 3)])
def test_work_of_tangents(native, n, vocab, dim):
    def asked(**kw):
        a, b = native.mf_embed_args(n_rows=n, vocab=vocab, dim=dim, **kw), C.c_size_t()
        assert native.lib().mf_embed_work_bytes(C.byref(a), C.byref(b)) == 0
        return b.value
    both = asked(dyd=4096, dEd=8192)
    assert asked(dEd=8192) == asked(dyd=4096) == both == native.mf_embed_work_bytes(n, vocab, dim, True)
    assert asked() == native.mf_embed_work_bytes(n, vocab, dim) <= both
