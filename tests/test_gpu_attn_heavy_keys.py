"""Forward tangents of rows in which a few keys outweigh the rest, as the first tokens of a sequence do, where
the tangents of the scores of the rest have a part in common: the worst cases of roundings to bf16
with P (*) S' as large as it is (attn_ops_util, attn_window_util), no larger than that."""
import math

import pytest

import attn_ops_util as au
import attn_window_util as wu
from gpu_util import need_gpu


def data(torch, lens, D, lead, score, apart, at=0):
    """Keys of which `lead` from the sequence's place `at` on score higher by `score`, and whose S' are those
    of the others less `apart`."""
    v = au.data(lens, 0, 1, 1, D, True, seed=76)
    g = torch.Generator().manual_seed(77)
    u = torch.randn(D, generator=g)
    u /= u.norm()
    first = torch.cat([torch.arange(n) - at for n in lens])[:, None]
    first = (first >= 0) & (first < lead)
    v["q"] = (v["q"].float() + 6 * u).bfloat16()
    v["k"] = (v["k"].float() + first * (score * math.sqrt(D) / 6) * u).bfloat16()
    v["kd"] = (v["kd"].float() + ~first * (apart * math.sqrt(D) / 6) * u).bfloat16()
    v["vd"] = (0.1 * v["vd"].float()).bfloat16()
    return v


@pytest.mark.gpu
@pytest.mark.parametrize("lens,window,sinks", [([1024], 2000, 0), ([40, 900], 2000, 0), ([1500], 1000, 4), ([70, 1200], 300, 1),
                                               ([3, 64, 700], 129, 16), ([900], 64, 1)])
@pytest.mark.parametrize("lead", [1, 4, 16])
@pytest.mark.parametrize("score,apart", [(0, 30), (6, 30), (12, 30), (9, 4), (3, 4)])
@pytest.mark.parametrize("D", [64, 40])
def test_tangents_of_heavy_first_keys(lens, window, sinks, lead, score, apart, D):
    torch, native = need_gpu()
    n = sum(lens)
    w = {k: t.cuda() for k, t in data(torch, lens, D, lead, score, apart).items()}
    ref, bound = wu.reference(w, lens, 1, 1, D, min(window, n), sinks)
    out = wu.run(native, w, lens, 1, 1, D, window, sinks)
    torch.cuda.synchronize()
    au.check(out, ref, bound, n, True)


@pytest.mark.gpu
@pytest.mark.parametrize("lens,window,sinks", [([1024], 1000, 0), ([1024], 500, 4), ([40, 900], 300, 1)])
@pytest.mark.parametrize("at,lead", [(70, 1), (100, 1), (300, 4)])
@pytest.mark.parametrize("score,apart", [(4, 30), (6, 30), (8, 30), (6, 4), (12, 4)])
def test_window_tangents_of_heavy_keys_on_the_way(lens, window, sinks, at, lead, score, apart):
    """Keys that outweigh what came before them, by less than moves the row's maximum, and by more."""
    torch, native = need_gpu()
    n = sum(lens)
    w = {k: t.cuda() for k, t in data(torch, lens, 64, lead, score, apart, at).items()}
    ref, bound = wu.reference(w, lens, 1, 1, 64, window, sinks)
    out = wu.run(native, w, lens, 1, 1, 64, window, sinks)
    torch.cuda.synchronize()
    au.check(out, ref, bound, n, True)
