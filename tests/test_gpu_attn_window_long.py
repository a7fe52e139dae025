"""Windowed attention on both sides of the sizes where its kernels' forms change: tiles of 128 keys
where all CTAs have a place and the window is 512 and longer, more CTAs a group from windows of 2048 on."""
import pytest

import attn_ops_util as au
import attn_window_util as wu
from gpu_util import need_gpu

CASES = {
    # lens, tail, Hq, Hkv, D, window, sinks
    "border_below": ([900, 400], 3, 4, 2, 64, 511, 4),
    "border": ([900, 400], 3, 4, 2, 64, 512, 4),
    "many_ctas": ([2000, 450], 0, 16, 1, 64, 600, 4),
    "narrow": ([30, 1, 0, 1500, 777], 9, 2, 1, 24, 700, 0),
    "odd": ([1000, 1000, 999], 0, 2, 2, 40, 899, 1),
    "all_sinks": ([1111, 650], 5, 3, 1, 64, 512, 128),
    "short_sequences": ([100] * 12, 0, 4, 4, 64, 600, 3),
    "thousands": ([3100], 0, 2, 1, 64, 2048, 5),
    "thousands_below": ([3100], 0, 2, 1, 64, 2047, 5),
    "thousands_group": ([2500, 600], 1, 6, 1, 64, 2200, 0),
}


@pytest.mark.gpu
@pytest.mark.parametrize("dual", [False, True])
@pytest.mark.parametrize("name", list(CASES))
def test_long_window_against_definition(name, dual):
    torch, native = need_gpu()
    lens, tail, Hq, Hkv, D, window, sinks = CASES[name]
    v = au.data(lens, tail, Hq, Hkv, D, dual, seed=73)
    ref, bound = wu.reference({k: t.cuda() for k, t in v.items()}, lens, Hq, Hkv, D, window, sinks)
    out = wu.run(native, au.wide(v), lens, Hq, Hkv, D, window, sinks)
    torch.cuda.synchronize()
    au.check(out, ref, bound, sum(lens), dual)
    torch.cuda.empty_cache()


@pytest.mark.gpu
@pytest.mark.parametrize("dual", [False, True])
def test_long_window_of_a_larger_batch(dual):
    """Sequences shorter than the window, in a batch with several CTAs a group: mf_attn_*'s results but for
    the order of sums and the tiles.  Either's outputs are off from 64 bits by 0.0042 in relative L2 at
    most (two keys a row; attn_rms_util), an lse by 2^-17 (1 + scale |q| |k|) and rbar by that of |S'| too:
    scale |q| |k| is 5 in the mean here and stays below 12, |S'| below 6."""
    torch, native = need_gpu()
    lens, Hq, Hkv, D = [1500, 1200, 1400], 8, 2, 64
    v = au.wide(au.data(lens, 2, Hq, Hkv, D, dual, seed=74))
    n = sum(lens)
    out = wu.run(native, v, lens, Hq, Hkv, D, 2100, 0)
    want = au.run(native, v, lens, Hq, Hkv, D)
    torch.cuda.synchronize()
    for k in au.names(dual):
        if k in ("lse", "rbar"):
            off = au.FLOAT * 13 * (1 if k == "lse" else 1 + 2 * 6)
            assert (out[k][:, :n] - want[k][:, :n]).abs().max() <= 2 * off, k
            continue
        a, b = out[k][:n].double(), want[k][:n].double()
        assert (a - b).norm() <= 2 * 0.0042 * b.norm(), k
