"""Windowed packed attention without a GPU: refusals, workspaces, the float64 definition."""
import ctypes as C

import pytest
import torch

import attn_ops_util as au
import attn_window_util as wu
from oracle import packed as op
from test_ops_cpu import ATTN_BAD, ATTN_BWD_BAD, DUAL, INVALID, OK, UNSUPPORTED, _attn, native  # noqa: F401


@pytest.mark.parametrize("kw", ATTN_BAD, ids=str)
def test_window_refuses(native, kw):  # noqa: F811
    for f in ("mf_attn_window_fwd", "mf_attn_window_bwd"):
        assert getattr(native.lib(), f)(C.byref(_attn(native, **kw)), 4, 1, None) == INVALID, f


@pytest.mark.parametrize("kw", ATTN_BWD_BAD, ids=str)
def test_window_backward_refuses(native, kw):  # noqa: F811
    assert native.lib().mf_attn_window_bwd(C.byref(_attn(native, **kw)), 4, 1, None) == INVALID


def test_window_refuses_windows_and_sinks(native):  # noqa: F811
    L = native.lib()
    for f in (L.mf_attn_window_fwd, L.mf_attn_window_bwd):
        for window, sinks in ((0, 0), (-1, 4), (-2 ** 40, 0), (4, -1)):
            assert f(C.byref(_attn(native)), window, sinks, None) == INVALID
        assert f(C.byref(_attn(native)), 4, 129, None) == UNSUPPORTED
        assert f(None, 4, 0, None) == INVALID
        assert f(C.byref(_attn(native, n_rows=0, q=None)), 4, 2, None) == OK
        assert f(C.byref(_attn(native, head_dim=72, ldq=512, ldk=512, ldv=512, ldo=512, lddo=512, lddq=512,
                               lddk=512, lddv=512, **DUAL)), 4, 2, None) == UNSUPPORTED


def test_window_work_bytes(native):  # noqa: F811
    """D of every row and head, and behind it the sums of sinks where there are chunks of query rows
    besides the first."""
    f = native.mf_attn_window_work_bytes
    assert f(10, 3, 1, 64, 4, 5) == 120 + 8
    assert f(512, 4, 2, 64, 4, 5) == 512 * 4 * 4
    assert f(513, 4, 2, 64, 4, 0) == 513 * 4 * 4
    sums = 2 * 2 * 2 * 2 * 5 * 64 * 4
    assert f(513, 4, 2, 64, 4, 5) == 513 * 4 * 4 + sums
    assert f(513, 4, 2, 64, 4, 5, True) == 2 * (513 * 4 * 4 + sums)
    assert f(513, 4, 2, 72, 4, 5) == 513 * 4 * 4 + 2 * sums
    assert f(513, 4, 2, 64, 513, 5) == native.mf_attn_work_bytes(513, 4)
    for bad in ((-1, 4, 2, 64, 4, 5), (513, 4, 2, 64, 0, 5), (513, 4, 2, 64, 4, -1), (513, 4, 2, 63, 4, 1),
                (513, 4, 2, 64, 4, 129)):
        with pytest.raises(native.MixflowError):
            f(*bad)
    a = _attn(native, n_rows=600, work_bytes=600 * 4 * 4)
    assert native.lib().mf_attn_window_bwd(C.byref(a), 4, 1, None) == INVALID


def test_pairs_and_definition():
    """The pairs by their words, and a window of everything against the causal definition."""
    lens, W, S = [5, 0, 1, 7], 3, 2
    pairs = op.window_pairs(lens, W, S)
    lo = 0
    want = torch.zeros(13, 13, dtype=torch.bool)
    for n in lens:
        for i in range(n):
            for j in range(i + 1):
                want[lo + i, lo + j] = i - j < W or j < S
        lo += n
    assert torch.equal(pairs, want)
    v = au.data(lens, 0, 2, 1, 8, False, seed=1)
    a = op.attention(*(v[k].double() for k in "qkv"), 2, 1, 8, lens, 0.3)
    b = op.masked_attention(*(v[k].double() for k in "qkv"), 2, 1, 8, op.window_pairs(lens, 7, 0), 0.3)
    for x, y in zip(a, b):
        assert (x - y).abs().max() < 1e-13


@pytest.mark.parametrize("dual", [False, True])
def test_bounds_are_those_of_all_pairs(dual):
    """With a window of everything the reference is attn_ops_util's, and no bound is above its (those
    take the largest error of all of a sequence's scores where these take a row's own)."""
    lens, Hq, Hkv, D = [40, 1, 23], 4, 2, 16
    v = au.data(lens, 2, Hq, Hkv, D, dual, seed=3)
    (r, b), (rw, bw) = au.reference(v, lens, Hq, Hkv, D), wu.reference(v, lens, Hq, Hkv, D, 100, 0)
    assert r.keys() == rw.keys() == bw.keys()
    for k in r:
        assert (r[k] - rw[k]).abs().max() < 1e-10, k
        assert (bw[k] - b[k]).max() < 1e-10, k
        assert k in ("od", "rbar", "dqd", "dkd", "dvd") or (bw[k] - b[k]).abs().max() < 1e-10, k
