"""Inputs, float64 reference and derived error bounds of the packed attention's tests."""
import math

import numpy as np
import torch

from oracle import packed as op

HALF = 2.0 ** -8          # bf16: half a step relative to the value
FLOAT = 2.0 ** -17        # float32 arithmetic: exponentials, sums, statistics, of the terms
# Relative bounds hold for normal numbers.  Below 2^-126 float32 and bf16 have a fixed step or
# flush to zero: a probability is then off by up to 2^-126, and the sums of at most 700 such
# terms times values below 2^6 that an output is made of by less than 2^-126 * 2^10 * 2^6.
TINY = 2.0 ** -110


def data(lens, tail, Hq, Hkv, D, dual, seed=0, qstd=1.0):
    g = torch.Generator().manual_seed(seed)
    N = sum(lens) + tail

    def rnd(cols, std):
        return (torch.randn(N, cols, generator=g) * std).to(torch.bfloat16)

    v = dict(q=rnd(Hq * D, qstd), k=rnd(Hkv * D, 1.0), v=rnd(Hkv * D, 1.0), do=rnd(Hq * D, 1.0))
    if dual:
        v.update(qd=rnd(Hq * D, 0.5), kd=rnd(Hkv * D, 0.5), vd=rnd(Hkv * D, 0.5), dod=rnd(Hq * D, 0.5))
    return v


def starts_of(lens):
    return torch.from_numpy(np.concatenate([[0], np.cumsum(lens)]).astype(np.int32))


def reference(v, lens, Hq, Hkv, D, scale=None):
    """Outputs in float64 and, for each, how far a kernel may be off that rounds P, P (*) S',
    dS, their tangents and its outputs to bf16 (HALF each, relative) and does everything else
    in float32 (FLOAT of the magnitudes summed)."""
    n, G = sum(lens), Hq // Hkv
    scale = scale or D ** -0.5
    dual = "qd" in v
    z = {k: t[:n].double() for k, t in v.items()}
    f = lambda q, k, w: op.attention(q, k, w, Hq, Hkv, D, lens, scale)
    prim = (z["q"], z["k"], z["v"])
    r = {}
    if dual:
        tang = (z["qd"], z["kd"], z["vd"])
        (r["o"], r["lse"]), (r["od"], r["rbar"]) = torch.func.jvp(f, prim, tang)
        g, gd = op.grads_dual(lambda *p: f(*p)[0], prim, z["do"], tang, z["dod"])
        r.update(dqd=gd[0], dkd=gd[1], dvd=gd[2])
    else:
        r["o"], r["lse"] = f(*prim)
        g = op.grads(lambda *p: f(*p)[0], prim, z["do"])
    r.update(dq=g[0], dk=g[1], dv=g[2])

    b = {k: torch.zeros_like(t) for k, t in r.items()}
    a = 0
    for m in lens:
        s = slice(a, a + m)
        a += m
        if not m:
            continue
        hd = lambda t, H: t[s].unflatten(1, (H, D)).transpose(0, 1)
        kv = lambda t: hd(t, Hkv).repeat_interleave(G, 0)
        Q, K, V, dO, O = hd(z["q"], Hq), kv(z["k"]), kv(z["v"]), hd(z["do"], Hq), hd(r["o"], Hq)
        S = (scale * Q @ K.mT).masked_fill(torch.ones(m, m, dtype=torch.bool).triu(1), -math.inf)
        P = torch.exp(S - r["lse"][:, s, None])
        # scores carry FLOAT of their terms' magnitudes, which moves P relatively
        eS = FLOAT * (1 + scale * Q.abs() @ K.abs().mT)
        E = HALF + eS                               # relative error of P as an operand
        low = torch.ones(m, m).tril()
        eO = (P * E) @ V.abs()
        put = lambda name, e, H: b[name].__setitem__(s, e.transpose(0, 1).flatten(1))
        own = lambda name, H: hd(r[name], H).abs() * HALF
        sumg = lambda e: e.unflatten(0, (Hkv, G)).sum(1)
        put("o", eO + own("o", Hq), Hq)
        b["lse"][:, s] = eS.masked_fill(low == 0, 0).amax(-1) + FLOAT * r["lse"][:, s].abs()
        dP = dO @ V.mT
        X = dP - (dO * O).sum(-1, keepdim=True)
        dS = P * X
        # D is formed from the rounded o
        eD = (dO.abs() * (eO + HALF * O.abs())).sum(-1, keepdim=True)
        edS = P * eD + dS.abs() * E + P * FLOAT * (dO.abs() @ V.abs().mT)
        put("dv", sumg((P * E).mT @ dO.abs()) + own("dv", Hkv), Hkv)
        put("dq", scale * edS @ K.abs() + own("dq", Hq), Hq)
        put("dk", scale * sumg(edS.mT @ Q.abs()) + own("dk", Hkv), Hkv)
        if not dual:
            continue
        Qd, Kd, Vd, dOd, Od = hd(z["qd"], Hq), kv(z["kd"]), kv(z["vd"]), hd(z["dod"], Hq), hd(r["od"], Hq)
        Sd = scale * (Qd @ K.mT + Q @ Kd.mT) * low
        rb = r["rbar"][:, s, None]
        eSd = FLOAT * scale * (Qd.abs() @ K.abs().mT + Q.abs() @ Kd.abs().mT) * low
        eR = (P * (eSd + eS * Sd.abs())).sum(-1, keepdim=True) + eS.amax(-1, keepdim=True) * rb.abs()
        eT = (P * (Sd.abs() * E + eSd)) @ V.abs() + (P * E) @ Vd.abs()
        eOd = eT + rb.abs() * eO + eR * O.abs()
        put("od", eOd + own("od", Hq), Hq)
        b["rbar"][:, s] = eR.squeeze(-1) + FLOAT * rb.squeeze(-1).abs()
        Pd = P * (Sd - rb)
        ePd = Pd.abs() * E + P * (eSd + eR)
        Xd = dOd @ V.mT + dO @ Vd.mT - (dOd * O + dO * Od).sum(-1, keepdim=True)
        eDd = (dOd.abs() * (eO + HALF * O.abs()) + dO.abs() * (eOd + HALF * Od.abs())).sum(-1, keepdim=True)
        dSd = Pd * X + P * Xd
        edSd = HALF * dSd.abs() + (ePd - HALF * Pd.abs()) * X.abs() + Pd.abs() * eD + P * eDd \
            + eS * (P * Xd).abs() + P * FLOAT * (dOd.abs() @ V.abs().mT + dO.abs() @ Vd.abs().mT) \
            + Pd.abs() * FLOAT * (dO.abs() @ V.abs().mT)
        put("dvd", sumg(ePd.mT @ dO.abs() + (P * E).mT @ dOd.abs()) + own("dvd", Hkv), Hkv)
        put("dqd", scale * (edSd @ K.abs() + edS @ Kd.abs()) + own("dqd", Hq), Hq)
        put("dkd", scale * sumg(edSd.mT @ Q.abs() + edS.mT @ Qd.abs()) + own("dkd", Hkv), Hkv)
    return r, {k: e + TINY for k, e in b.items()}


MARK = -7.0


def run(native, v, lens, Hq, Hkv, D, scale=0.0, backward=True, starts=None, stream=None, out=None):
    """Both passes on the GPU, from column ranges of wider rows into column ranges of rows that
    are filled with a mark; returns the outputs (all rows)."""
    dual = "qd" in v
    N = v["q"].shape[0]
    bf = torch.bfloat16
    if out is None:
        out = {}
        for k, H in (("o", Hq), ("od", Hq), ("dq", Hq), ("dk", Hkv), ("dv", Hkv), ("dqd", Hq),
                     ("dkd", Hkv), ("dvd", Hkv)):
            out[k] = torch.full((N, H * D + 8), MARK, dtype=bf, device="cuda")[:, 8:]
        out["lse"], out["rbar"] = (torch.full((Hq, N), MARK, device="cuda") for _ in range(2))
        out["work"] = torch.empty(native.mf_attn_work_bytes(N, Hq, dual), dtype=torch.uint8, device="cuda")
        out["status"] = torch.zeros(1, dtype=torch.int32, device="cuda")
    t = lambda *names: {n: out[n] for n in names} if dual else {}
    kw = dict(n_heads=Hq, n_kv_heads=Hkv, head_dim=D, scale=scale, status=out["status"], stream=stream,
              seq_start=starts_of(lens).cuda() if starts is None else starts,
              **({k: v[k] for k in ("qd", "kd", "vd")} if dual else {}), **t("od", "rbar"))
    native.mf_attn_fwd(v["q"], v["k"], v["v"], out["o"], out["lse"], **kw)
    if backward:
        native.mf_attn_bwd(v["q"], v["k"], v["v"], out["o"], out["lse"], v["do"], out["dq"], out["dk"],
                           out["dv"], work=out["work"], dod=v.get("dod"), **t("dqd", "dkd", "dvd"), **kw)
    return out


def wide(v):
    """The inputs as column ranges of one buffer of rows, as a fused projection leaves them."""
    out = {}
    for names in (("q", "k", "v"), ("qd", "kd", "vd"), ("do",), ("dod",)):
        if names[0] in v:
            cols = [v[n].shape[1] for n in names]
            x = torch.cat([v[n] for n in names] + [torch.full((v["q"].shape[0], 8), math.nan, dtype=torch.bfloat16)], 1).cuda()
            out.update(zip(names, x.split(cols + [8], 1)))
    return out


def names(dual, backward=True):
    r = ["o", "lse"] + ["od", "rbar"] * dual
    return r + (["dq", "dk", "dv"] + ["dqd", "dkd", "dvd"] * dual) * backward


def check(out, ref, bound, n, dual, backward=True):
    assert int(out["status"].item()) == 0
    for k in names(dual, backward):
        x = out[k].double().cpu()
        stat = k in ("lse", "rbar")
        got, rest = (x[:, :n], x[:, n:]) if stat else (x[:n], x[n:])
        assert (rest == MARK).all(), k
        if not n:
            continue
        assert torch.isfinite(got).all(), k
        off = (got - ref[k]).abs()
        worst = (off - bound[k]).max().item()
        assert worst <= 0, (k, worst, off.max().item(), bound[k].max().item())
        # a kernel's roundings have random signs: together they stay well inside the sum of
        # their largest sizes
        if n > 200 and not stat:
            assert off.norm() <= 0.5 * bound[k].norm(), (k, off.norm().item(), bound[k].norm().item())
