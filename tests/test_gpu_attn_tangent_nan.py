"""Values that are not finite in tangents reach tangents alone: o, lse, dq, dk, dv do not depend on
q', k', v', do'."""
import math

import pytest

import attn_ops_util as au
from gpu_util import need_gpu


@pytest.mark.gpu
@pytest.mark.parametrize("D", [64, 40])
@pytest.mark.parametrize("which", ["qd", "kd", "vd", "dod"])
@pytest.mark.parametrize("value", [math.nan, math.inf])
def test_tangents_stay_among_themselves(which, D, value):
    torch, native = need_gpu()
    lens, tail, Hq, Hkv = [70, 45, 100, 200], 33, 4, 2
    n = sum(lens)
    v = au.data(lens, tail, Hq, Hkv, D, True, seed=41)
    want = {k: t.clone() for k, t in au.run(native, au.wide(v), lens, Hq, Hkv, D).items()}
    # rows in tiles on a sequence's border and inside one, and behind the last sequence
    v[which][[3, 90, 116, 219, 350, n + 2]] = value
    out = au.run(native, au.wide(v), lens, Hq, Hkv, D)
    torch.cuda.synchronize()
    assert int(out["status"].item()) == 0
    for k in ("o", "lse", "dq", "dk", "dv"):
        assert torch.equal(out[k], want[k]), (k, (out[k] != want[k]).nonzero()[:4].tolist())
    # and they do show among the tangents: in the rows that attend to such a row
    seen = {"qd": "od", "kd": "od", "vd": "od", "dod": "dvd"}[which]
    assert not torch.isfinite(out[seen][[3, 90, 116, 219]]).all(1).any()
    clear = [r for r in range(n) if r < 3 or 70 <= r < 90 or r in (115, *range(215, 219))]
    if which != "dod":
        assert torch.equal(out["od"][clear], want["od"][clear])
        assert torch.equal(out["dqd"][clear], want["dqd"][clear])
