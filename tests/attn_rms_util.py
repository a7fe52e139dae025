"""Expected sizes of the packed attention's errors, and a float64 emulation of its roundings.

The bounds of attn_ops_util are worst cases: sums of the largest roundings.  These are variances.
A rounding to bf16 is off by a uniform part of a step, at most 2^-8 of the value each way, so its
relative variance is at most U = 2^-16 / 3; roundings are independent, so variances add up, where
one error enters many terms (D, D') as the square of its sum.  A tensor's error in the 2-norm is
then the root of the sum of its variances, up to a few per cent for thousands of elements, and
the largest of float32's own errors (2^-17 of the terms, attn_ops_util.FLOAT) are below a tenth of
that.  SLACK covers both.

The forward tangent is o' = sum P (S' - rbar) v + P v'.  The kernels round P (S' - c), with c a mean
of the row's own S' over some of its keys, so |S' - c| <= |S' - rbar| + max |S' - rbar|: what is
rounded does not grow with a part that all of a row's S' have in common."""
import math

import torch

import attn_ops_util as au
from oracle import packed as op

U = 2.0 ** -16 / 3
SLACK = 1.25


def shifted(lens, tail, Hq, Hkv, D, dual, seed, offset):
    """au.data with a common part in every key, `offset` of a vector of unit variance: scores of a
    row move together, and so do their tangents, by q' times that vector."""
    v = au.data(lens, tail, Hq, Hkv, D, dual, seed=seed)
    g = torch.Generator().manual_seed(seed + 1000)
    mu = torch.randn(1, Hkv * D, generator=g)
    v["k"] = (v["k"].float() + offset * mu).to(torch.bfloat16)
    return v


def _parts(v, lens, Hq, Hkv, D):
    """Each sequence's rows and its tensors as [heads][rows][D], keys and values a query head."""
    G, a = Hq // Hkv, 0
    for m in lens:
        s = slice(a, a + m)
        a += m
        if not m:
            continue
        t = {}
        for k, x in v.items():
            H = Hkv if k in ("k", "v", "kd", "vd") else Hq
            y = x[s].double().unflatten(1, (H, D)).transpose(0, 1)
            t[k] = y.repeat_interleave(G, 0) if H == Hkv else y
        yield s, t, torch.ones(m, m, dtype=torch.bool).tril()


def variances(v, lens, Hq, Hkv, D, scale=None):
    """The largest expected square of each output's error, elementwise."""
    n, G, dual = sum(lens), Hq // Hkv, "qd" in v
    scale = scale or D ** -0.5
    r, _ = au.reference(v, lens, Hq, Hkv, D, scale)
    var = {k: torch.zeros_like(t) for k, t in r.items()}
    sq = lambda t: t * t
    sumg = lambda e: e.unflatten(0, (Hkv, G)).sum(1)
    for s, t, low in _parts({k: x[:n] for k, x in v.items()}, lens, Hq, Hkv, D):
        hd = lambda x, H: x[s].unflatten(1, (H, D)).transpose(0, 1)
        put = lambda name, e, H: var[name].__setitem__(s, (e + U * sq(hd(r[name], H))).transpose(0, 1).flatten(1))
        Q, K, V, dO, O = t["q"], t["k"], t["v"], t["do"], hd(r["o"], Hq)
        S = (scale * Q @ K.mT).masked_fill(~low, -math.inf)
        P = torch.exp(S - r["lse"][:, s, None])
        ep = U * sq(P) @ sq(V)                       # of P v
        put("o", ep, Hq)
        vo = ep + U * sq(O)
        X = dO @ V.mT - (dO * O).sum(-1, keepdim=True)
        dS = P * X
        vD = sq(dO) @ vo.mT                          # D of row i from the rounded o of row i
        vD = torch.diagonal(vD, dim1=-2, dim2=-1)[..., None]
        PK = P @ K
        put("dv", sumg(U * sq(P).mT @ sq(dO)), Hkv)
        put("dq", sq(torch.tensor(scale)) * (vD * sq(PK) + U * sq(dS) @ sq(K)), Hq)
        put("dk", scale ** 2 * sumg((vD * sq(P)).mT @ sq(Q) + U * sq(dS).mT @ sq(Q)), Hkv)
        if not dual:
            continue
        Qd, Kd, Vd, dOd, Od = t["qd"], t["kd"], t["vd"], t["dod"], hd(r["od"], Hq)
        Sd = scale * (Qd @ K.mT + Q @ Kd.mT)
        rb = r["rbar"][:, s, None]
        near = (Sd - rb).abs() * low
        far = near.amax(-1, keepdim=True)
        eod = U * sq(P * (near + far)) @ sq(V) + U * sq(P) @ sq(Vd) + sq(far) * ep
        put("od", eod, Hq)
        vod = eod + U * sq(Od)
        Pd = P * (Sd - rb)
        Xd = dOd @ V.mT + dO @ Vd.mT - (dOd * O + dO * Od).sum(-1, keepdim=True)
        dSd = Pd * X + P * Xd
        vDd = 2 * (sq(dOd) * vo).sum(-1, keepdim=True) + 2 * (sq(dO) * vod).sum(-1, keepdim=True)
        put("dvd", sumg(U * (sq(Pd).mT @ sq(dO) + sq(P).mT @ sq(dOd))), Hkv)
        put("dqd", scale ** 2 * (2 * vDd * sq(PK) + 2 * vD * sq(Pd @ K + P @ Kd)
                                 + U * (sq(dSd) @ sq(K) + sq(dS) @ sq(Kd))), Hq)
        put("dkd", scale ** 2 * sumg(2 * (vDd * sq(P)).mT @ sq(Q) + 2 * (vD * sq(Pd)).mT @ sq(Q)
                                     + 2 * (vD * sq(P)).mT @ sq(Qd)
                                     + U * (sq(dSd).mT @ sq(Q) + sq(dS).mT @ sq(Qd))), Hkv)
    return r, var


def bounds(v, lens, Hq, Hkv, D, scale=None):
    """au.reference, its worst cases of o' (and so of D', dq', dk') with P (S' - c) rounded: c may lie
    as far from rbar as the row's furthest S', which an element whose own S' is small can feel."""
    n, G = sum(lens), Hq // Hkv
    scale = scale or D ** -0.5
    r, b = au.reference(v, lens, Hq, Hkv, D, scale)
    if "qd" not in v:
        return r, b
    for s, t, low in _parts({k: x[:n] for k, x in v.items()}, lens, Hq, Hkv, D):
        hd = lambda x, H: x[s].unflatten(1, (H, D)).transpose(0, 1)
        flat = lambda x: x.transpose(0, 1).flatten(1)
        Q, K, V, Vd, dO, Od = t["q"], t["k"], t["v"], t["vd"], t["do"], hd(r["od"], Hq)
        S = (scale * Q @ K.mT).masked_fill(~low, -math.inf)
        P = torch.exp(S - r["lse"][:, s, None])
        near = (scale * (t["qd"] @ K.mT + Q @ t["kd"].mT) - r["rbar"][:, s, None]).abs() * low
        far = near.amax(-1, keepdim=True)
        E = au.HALF + au.FLOAT * (1 + scale * Q.abs() @ K.abs().mT)
        eSd = au.FLOAT * scale * (t["qd"].abs() @ K.abs().mT + Q.abs() @ t["kd"].abs().mT) * low
        e = (P * ((near + far) * E + eSd)) @ V.abs() + (P * E) @ Vd.abs() + far * ((P * E) @ V.abs())
        more = (e + au.HALF * Od.abs() - hd(b["od"], Hq)).clamp_min(0)
        b["od"][s] += flat(more)
        eD = (dO.abs() * more).sum(-1, keepdim=True)
        b["dqd"][s] += flat(scale * (P * eD) @ K.abs())
        b["dkd"][s] += flat(scale * ((P * eD).mT @ Q.abs()).unflatten(0, (Hkv, G)).sum(1))
    return r, b


def check_norms(out, r, var, n):
    """Every rounded output's error in the 2-norm against its expected size."""
    for k, x in var.items():
        if k in ("lse", "rbar"):
            continue
        off = (out[k][:n].double().cpu() - r[k]).norm().item()
        most = SLACK * x.sum().sqrt().item()
        assert off <= most, (k, off, most, off / r[k].norm().item())


def emulate(v, lens, Hq, Hkv, D, scale=None, centre=True, drop=()):
    """The operators in float64 with the kernels' roundings to bf16.  centre False: P (*) S' is
    rounded as it is; drop: terms left out, as a mistake would."""
    n, G, dual = sum(lens), Hq // Hkv, "qd" in v
    scale = scale or D ** -0.5
    r16 = lambda t: t.to(torch.float32).bfloat16().double()
    out = {k: torch.zeros(n, Hq * D, dtype=op.F64) for k in ("o", "dq") + ("od", "dqd") * dual}
    out.update({k: torch.zeros(n, Hkv * D, dtype=op.F64) for k in ("dk", "dv") + ("dkd", "dvd") * dual})
    out.update({k: torch.zeros(Hq, n, dtype=op.F64) for k in ("lse",) + ("rbar",) * dual})
    sumg = lambda e: e.unflatten(0, (Hkv, G)).sum(1)
    for s, t, low in _parts({k: x[:n] for k, x in v.items()}, lens, Hq, Hkv, D):
        put = lambda name, e: out[name].__setitem__(s, r16(e).transpose(0, 1).flatten(1))
        Q, K, V, dO = t["q"], t["k"], t["v"], t["do"]
        S = (scale * Q @ K.mT).masked_fill(~low, -math.inf)
        p = torch.exp(S - S.amax(-1, keepdim=True))
        l = p.sum(-1, keepdim=True)
        lse = S.amax(-1, keepdim=True) + torch.log(l)
        out["lse"][:, s] = lse.squeeze(-1)
        acc = r16(p) @ V / l
        put("o", acc)
        O = r16(acc)
        P = torch.exp(S - lse)
        X = dO @ V.mT - (dO * O).sum(-1, keepdim=True)
        dS = r16(P * X)
        put("dv", sumg(r16(P).mT @ dO))
        put("dq", scale * dS @ K)
        put("dk", scale * sumg(dS.mT @ Q))
        if not dual:
            continue
        Qd, Kd, Vd, dOd = t["qd"], t["kd"], t["vd"], t["dod"]
        Sd = scale * (Qd @ K.mT + Q @ Kd.mT) * low
        rb = (p * Sd).sum(-1, keepdim=True) / l
        out["rbar"][:, s] = rb.squeeze(-1)
        c = Sd[..., :64].sum(-1, keepdim=True) / low[:, :64].sum(-1, keepdim=True) if centre else 0 * rb
        od = (r16(p * (Sd - c)) @ V + r16(p) @ Vd * ("od" not in drop)) / l - (rb - c) * acc
        put("od", od)
        Od = r16(od)
        Pd = P * (Sd - rb)
        Xd = dOd @ V.mT + dO @ Vd.mT - (dOd * O + dO * Od * ("dkd" not in drop)).sum(-1, keepdim=True)
        dSd = r16(Pd * X + P * Xd)
        put("dvd", sumg(r16(Pd).mT @ dO * ("dvd" not in drop) + r16(P).mT @ dOd))
        put("dqd", scale * (dSd @ K + dS @ Kd * ("dqd" not in drop)))
        put("dkd", scale * sumg(dSd.mT @ Q + dS.mT @ Qd))
    return out
