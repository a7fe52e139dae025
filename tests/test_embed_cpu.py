"""Embedding lookup and its gradient without a GPU: refusals of the C entry points and the binding,
workspaces."""
import ctypes as C
import math

import pytest
import torch


@pytest.fixture(scope="module")
def native():
    from paper_2505_00793_gb300 import build, native
    build.build()
    return native


OK, INVALID = 0, 1
P = 4096   # a pointer that no refused call reads


def _embed(native, **kw):
    a = native.mf_embed_args()
    a.n_rows, a.vocab, a.dim, a.e_prec, a.y_prec, a.scale = 40, 100, 24, 0, 1, 2.0
    for i, k in enumerate(("ids", "E", "y", "dy", "dE", "work")):
        setattr(a, k, P * (1 + i))
    a.ldE = a.ldy = a.lddy = a.lddE = 24
    a.work_bytes = 1 << 30
    for k, v in kw.items():
        setattr(a, k, v)
    return a


BOTH = [dict(n_rows=-1), dict(n_rows=2 ** 31), dict(vocab=0), dict(vocab=-4), dict(vocab=2 ** 31), dict(dim=0),
        dict(dim=2 ** 20 + 1), dict(y_prec=2), dict(scale=math.nan), dict(scale=math.inf), dict(ids=None),
        dict(n_seq=3), dict(n_seq=-1), dict(seq_start=P, n_seq=0)]
FWD = [dict(e_prec=-1), dict(E=None), dict(y=None), dict(E=P + 8), dict(y=3 * P + 2), dict(ldE=16), dict(ldE=26),
       dict(ldy=8), dict(ldy=-24), dict(Ed=P * 9), dict(yd=P * 9), dict(Ed=P * 9, yd=P * 10 + 4), dict(y=P * 2),
       dict(y=P), dict(Ed=P * 9, yd=3 * P), dict(Ed=P * 9, yd=P * 9)]
BWD = [dict(dy=None), dict(dE=None), dict(dy=4 * P + 8), dict(dE=5 * P + 4), dict(lddy=16), dict(lddE=20),
       dict(lddE=1 << 40), dict(dyd=P * 9), dict(dEd=P * 9), dict(work=None), dict(work=6 * P + 4),
       dict(work_bytes=15), dict(dE=4 * P), dict(dE=P), dict(work=4 * P), dict(dyd=P * 9, dEd=P * 5),
       dict(dyd=P * 9, dEd=P * 9)]


@pytest.mark.parametrize("kw", BOTH + FWD, ids=str)
def test_lookup_refuses(native, kw):
    assert native.lib().mf_embed_fwd(C.byref(_embed(native, **kw)), None) == INVALID


@pytest.mark.parametrize("kw", BOTH + BWD, ids=str)
def test_gradient_refuses(native, kw):
    assert native.lib().mf_embed_bwd(C.byref(_embed(native, **kw)), None) == INVALID


def test_calls_without_work(native):
    L = native.lib()
    assert L.mf_embed_fwd(None, None) == INVALID and L.mf_embed_bwd(None, None) == INVALID
    assert L.mf_embed_work_bytes(None, None) == INVALID
    assert L.mf_embed_fwd(C.byref(_embed(native, n_rows=0, ids=None, E=None, y=None, Ed=P)), None) == OK


def test_work_bytes(native):
    f = native.mf_embed_work_bytes
    sizes = [f(n, v, d, dual) for n, v, d, dual in
             ((0, 1, 1, False), (40, 100, 24, False), (40, 100, 24, True), (4096, 100, 24, True),
              (4096, 100, 1025, True), (4096, 10 ** 6, 1025, True), (10 ** 6, 10 ** 6, 1025, True))]
    assert sizes == sorted(sizes) and sizes[0] > 0
    # two lists of tokens at 8 bytes, and less than the rows themselves for the rest
    assert f(10 ** 6, 50000, 1024) < 10 ** 6 * 16 + 10 ** 6 * 1024 * 2
    for bad in ((-1, 4, 8), (4, 0, 8), (4, 4, 0), (4, 4, 2 ** 21), (2 ** 31, 4, 8)):
        with pytest.raises(native.MixflowError):
            f(*bad)
    a = _embed(native, work_bytes=f(40, 100, 24) - 1)
    assert native.lib().mf_embed_bwd(C.byref(a), None) == INVALID


def test_binding_refuses(native):
    ids, t = torch.zeros(4, dtype=torch.int32), torch.zeros(4, 8)
    with pytest.raises(ValueError, match="CUDA"):
        native.mf_embed_fwd(ids, t, t)
    with pytest.raises(ValueError, match="CUDA"):
        native.mf_embed_bwd(ids, t, t, torch.zeros(8))
