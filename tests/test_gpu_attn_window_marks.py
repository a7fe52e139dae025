"""Windowed attention with seq_start of wrong contents: nothing is written outside the outputs' rows and
columns, the statistics and the workspace.  Every output lies inside a larger marked buffer."""
import pytest

import attn_ops_util as au
from gpu_util import need_gpu

MARK = -7.0
STARTS = [[0, 200, 100, 1260], [5, -7, 10 ** 9, 2 ** 31 - 1], [0, 0, 0, -5], [1300, 1300, 1300, 1260],
          [600, 3, 1200, 1000], [-2 ** 31, 2 ** 31 - 1, -2 ** 31, 1260], [0, 1259, 513, 1260], [0, 511, 1, 1100],
          [1259, 1258, 700, 1260], [0, 512, 1024, 1260]]


def inside(torch, shape, dtype, before, value):
    """A contiguous view of a marked buffer, `before` elements behind its begin and as many before its end."""
    n = 1
    for x in shape:
        n *= x
    buf = torch.full((n + 2 * before,), value, dtype=dtype, device="cuda")
    return buf[before:before + n].view(shape), buf


@pytest.mark.gpu
@pytest.mark.parametrize("D,dual,Hq,Hkv", [(64, False, 2, 1), (64, True, 2, 1), (24, True, 3, 3), (128, False, 2, 1),
                                           (64, False, 6, 2), (64, False, 2, 2)])
@pytest.mark.parametrize("window,sinks", [(20, 100), (600, 128), (1, 3), (700, 0)])
def test_nothing_outside_is_written(D, dual, Hq, Hkv, window, sinks):
    torch, native = need_gpu()
    N = 1260
    v = au.wide(au.data([N], 0, Hq, Hkv, D, dual, seed=75))
    out, all_of = {}, {}
    for k, H in (("o", Hq), ("dq", Hq), ("dk", Hkv), ("dv", Hkv)):
        for t in ("", "d")[:1 + dual]:
            rows, all_of[k + t] = inside(torch, (N, H * D + 16), torch.bfloat16, 256 * (H * D + 16), MARK)
            out[k + t] = rows[:, 8:8 + H * D]
    for k in ("lse", "rbar")[:1 + dual]:
        out[k], all_of[k] = inside(torch, (Hq, N), torch.float32, 4096, MARK)
    size = native.mf_attn_window_work_bytes(N, Hq, Hkv, D, window, sinks, dual)
    work, all_of["work"] = inside(torch, (size,), torch.uint8, 1 << 20, 0x5a)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    names = lambda *ks: {k: out[k] for k in ks} if dual else {}
    tang = {k: v[k] for k in ("qd", "kd", "vd")} if dual else {}
    for s in STARTS:
        kw = dict(n_heads=Hq, n_kv_heads=Hkv, head_dim=D, window=window, n_sink=sinks, status=status,
                  seq_start=torch.tensor(s, dtype=torch.int32, device="cuda"), **tang, **names("od", "rbar"))
        native.mf_attn_window_fwd(v["q"], v["k"], v["v"], out["o"], out["lse"], **kw)
        native.mf_attn_window_bwd(v["q"], v["k"], v["v"], out["o"], out["lse"], v["do"], out["dq"], out["dk"], out["dv"],
                                  work=work, dod=v.get("dod"), **names("dqd", "dkd", "dvd"), **kw)
        torch.cuda.synchronize()
        assert int(status.item()) == 0
        for k, buf in all_of.items():
            n = {"work": 1 << 20, "lse": 4096, "rbar": 4096}.get(k)
            mark = 0x5a if k == "work" else MARK
            if n is None:
                wide = buf.view(-1, out[k].shape[1] + 16)
                assert (wide[:256] == mark).all() and (wide[256 + N:] == mark).all(), (k, s)
                assert (wide[:, :8] == mark).all() and (wide[:, -8:] == mark).all(), (k, s)
            else:
                assert (buf[:n] == mark).all() and (buf[-n:] == mark).all(), (k, s)
