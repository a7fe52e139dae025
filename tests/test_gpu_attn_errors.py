"""Sizes of the packed attention's errors against what its roundings make them (attn_rms_util):
long and short sequences, and keys with a common part, which all of a row's tangent scores then
have in common: it cancels in o', and must not be rounded before it does."""
import pytest

import attn_ops_util as au
import attn_rms_util as ar
from gpu_util import need_gpu

CASES = {
    # lens, tail, Hq, Hkv, D, common part of the keys
    "ragged": ([300, 1, 77], 2, 2, 1, 64, 0.0),
    "short": ([2] * 60 + [5, 3, 9, 1, 40], 0, 4, 2, 64, 0.0),
    "shifted_3": ([300, 77], 0, 2, 1, 64, 3.0),
    "shifted_30": ([300, 77], 5, 4, 2, 64, 30.0),
    "shifted_30_narrow": ([700, 20, 130], 0, 2, 2, 24, 30.0),
    # a sequence that has few keys in its row tile's first key tile
    "shifted_30_late": ([60, 200, 122, 2, 300], 0, 2, 1, 64, 30.0),
}


@pytest.mark.gpu
@pytest.mark.parametrize("dual", [False, True])
@pytest.mark.parametrize("name", list(CASES))
def test_errors_have_their_expected_size(name, dual):
    torch, native = need_gpu()
    lens, tail, Hq, Hkv, D, offset = CASES[name]
    v = ar.shifted(lens, tail, Hq, Hkv, D, dual, 31, offset)
    r, var = ar.variances(v, lens, Hq, Hkv, D)
    out = au.run(native, au.wide(v), lens, Hq, Hkv, D)
    torch.cuda.synchronize()
    assert int(out["status"].item()) == 0
    ar.check_norms(out, r, var, sum(lens))


@pytest.mark.gpu
def test_errors_of_wide_heads():
    torch, native = need_gpu()
    lens, Hq, Hkv, D = [300, 1, 77, 2, 2, 3], 4, 2, 128
    v = au.data(lens, 0, Hq, Hkv, D, False, seed=32)
    r, var = ar.variances(v, lens, Hq, Hkv, D)
    out = au.run(native, au.wide(v), lens, Hq, Hkv, D)
    torch.cuda.synchronize()
    ar.check_norms(out, r, var, sum(lens))


@pytest.mark.gpu
@pytest.mark.parametrize("grow", [6.0, 40.0])
def test_tangents_whose_scores_grow(grow):
    """Scores that grow along the sequence, so that the reference maximum of a row moves on the way
    and earlier sums are rescaled, and tangent scores with a common part of their own there."""
    torch, native = need_gpu()
    lens, Hq, Hkv, D = [400, 150], 2, 1, 64
    v = ar.shifted(lens, 0, Hq, Hkv, D, True, 33, 10.0)
    ramp = torch.cat([torch.arange(m) / m for m in lens])[:, None] * grow
    g = torch.Generator().manual_seed(34)
    way = torch.randn(1, D, generator=g)
    v["q"] = (0.2 * v["q"].float() + way.repeat(1, Hq)).bfloat16()
    v["k"] = (v["k"].float() + ramp * way / 8).bfloat16()
    r, var = ar.variances(v, lens, Hq, Hkv, D)
    _, bound = ar.bounds(v, lens, Hq, Hkv, D)
    out = au.run(native, au.wide(v), lens, Hq, Hkv, D)
    torch.cuda.synchronize()
    au.check(out, r, bound, sum(lens), True)
    ar.check_norms(out, r, var, sum(lens))


@pytest.mark.gpu
@pytest.mark.parametrize("lens,Hq,Hkv,D", [([145], 4, 2, 16), ([112, 100], 3, 1, 56), ([400, 245], 4, 2, 40),
                                           ([1, 129, 60, 900], 2, 1, 64)])
@pytest.mark.parametrize("std", [3.0, 8.0])
def test_tangents_of_sharp_rows(lens, Hq, Hkv, D, std):
    """Scores so wide that single keys take a row, wherever on the way they come."""
    torch, native = need_gpu()
    v = au.data(lens, 3, Hq, Hkv, D, True, seed=35, qstd=std)
    r, var = ar.variances(v, lens, Hq, Hkv, D)
    _, bound = ar.bounds(v, lens, Hq, Hkv, D)
    out = au.run(native, au.wide(v), lens, Hq, Hkv, D)
    torch.cuda.synchronize()
    au.check(out, r, bound, sum(lens), True)
    ar.check_norms(out, r, var, sum(lens))
