"""Float64 reference and derived error bounds of the windowed attention's tests, and its calls.  Inputs
and what a rounding is worth are attn_ops_util's; the bounds are its bounds over the pairs of rows
that attend to one another in place of all causal ones."""
import torch

import attn_ops_util as au
from attn_ops_util import FLOAT, HALF, MARK
from oracle import packed as op

# As attn_ops_util.TINY, for sums of up to 2^12 terms.
TINY = 2.0 ** -108


def reference(v, lens, Hq, Hkv, D, window, sinks, scale=None):
    """Outputs in float64 and, for each, how far a kernel may be off that rounds P, P (*) S', dS,
    their tangents and its outputs to bf16 (HALF each, relative) and does everything else in float32
    (FLOAT of the magnitudes summed).  On the inputs' device; results on the CPU."""
    n, G, dual = sum(lens), Hq // Hkv, "qd" in v
    scale = scale or D ** -0.5
    z = {k: t[:n].double() for k, t in v.items()}
    pairs = op.window_pairs(lens, window, sinks, v["q"].device)
    f = lambda q, k, w: op.masked_attention(q, k, w, Hq, Hkv, D, pairs, scale)
    prim = (z["q"], z["k"], z["v"])
    r, b = {}, {}
    if dual:
        tang = (z["qd"], z["kd"], z["vd"])
        (r["o"], r["lse"]), (r["od"], r["rbar"]) = torch.func.jvp(f, prim, tang)
        g, gd = op.grads_dual(lambda *p: f(*p)[0], prim, z["do"], tang, z["dod"])
        r.update(dqd=gd[0], dkd=gd[1], dvd=gd[2])
    else:
        r["o"], r["lse"] = f(*prim)
        g = op.grads(lambda *p: f(*p)[0], prim, z["do"])
    r.update(dq=g[0], dk=g[1], dv=g[2])

    hd = lambda t, H: t.unflatten(1, (H, D)).transpose(0, 1)
    kv = lambda t: hd(t, Hkv).repeat_interleave(G, 0)
    flat = lambda t: t.transpose(0, 1).flatten(1)
    sumg = lambda e: e.unflatten(0, (Hkv, G)).sum(1)

    def put(name, e, H):
        b[name] = flat(e + hd(r[name], H).abs() * HALF)

    Q, K, V, dO, O = hd(z["q"], Hq), kv(z["k"]), kv(z["v"]), hd(z["do"], Hq), hd(r["o"], Hq)
    S = (scale * Q @ K.mT).masked_fill(~pairs, -torch.inf)
    P = torch.exp(S - r["lse"][..., None])
    eS = FLOAT * (1 + scale * Q.abs() @ K.abs().mT)
    E = HALF + eS                               # relative error of P as an operand
    eO = (P * E) @ V.abs()
    put("o", eO, Hq)
    b["lse"] = eS.masked_fill(~pairs, 0).amax(-1) + FLOAT * r["lse"].abs()
    X = dO @ V.mT - (dO * O).sum(-1, keepdim=True)
    dS = P * X
    eD = (dO.abs() * (eO + HALF * O.abs())).sum(-1, keepdim=True)     # D is formed from the rounded o
    edS = P * eD + dS.abs() * E + P * FLOAT * (dO.abs() @ V.abs().mT)
    put("dv", sumg((P * E).mT @ dO.abs()), Hkv)
    put("dq", scale * edS @ K.abs(), Hq)
    put("dk", scale * sumg(edS.mT @ Q.abs()), Hkv)
    if dual:
        Qd, Kd, Vd, dOd, Od = hd(z["qd"], Hq), kv(z["kd"]), kv(z["vd"]), hd(z["dod"], Hq), hd(r["od"], Hq)
        Sd = scale * (Qd @ K.mT + Q @ Kd.mT) * pairs
        rb = r["rbar"][..., None]
        eSd = FLOAT * scale * (Qd.abs() @ K.abs().mT + Q.abs() @ Kd.abs().mT) * pairs
        eR = (P * (eSd + eS * Sd.abs())).sum(-1, keepdim=True) \
            + eS.masked_fill(~pairs, 0).amax(-1, keepdim=True) * rb.abs()
        eT = (P * (Sd.abs() * E + eSd)) @ V.abs() + (P * E) @ Vd.abs()
        eOd = eT + rb.abs() * eO + eR * O.abs()
        put("od", eOd, Hq)
        b["rbar"] = eR.squeeze(-1) + FLOAT * rb.squeeze(-1).abs()
        Pd = P * (Sd - rb)
        ePd = Pd.abs() * E + P * (eSd + eR)
        Xd = dOd @ V.mT + dO @ Vd.mT - (dOd * O + dO * Od).sum(-1, keepdim=True)
        eDd = (dOd.abs() * (eO + HALF * O.abs()) + dO.abs() * (eOd + HALF * Od.abs())).sum(-1, keepdim=True)
        dSd = Pd * X + P * Xd
        edSd = HALF * dSd.abs() + (ePd - HALF * Pd.abs()) * X.abs() + Pd.abs() * eD + P * eDd \
            + eS * (P * Xd).abs() + P * FLOAT * (dOd.abs() @ V.abs().mT + dO.abs() @ Vd.abs().mT) \
            + Pd.abs() * FLOAT * (dO.abs() @ V.abs().mT)
        put("dvd", sumg(ePd.mT @ dO.abs() + (P * E).mT @ dOd.abs()), Hkv)
        put("dqd", scale * (edSd @ K.abs() + edS @ Kd.abs()), Hq)
        put("dkd", scale * sumg(edSd.mT @ Q.abs() + edS.mT @ Qd.abs()), Hkv)
    return {k: t.cpu() for k, t in r.items()}, {k: (e + TINY).cpu() for k, e in b.items()}


def buffers(native, N, Hq, Hkv, D, window, sinks, dual):
    """Outputs as column ranges of rows filled with a mark."""
    out = {}
    for k, H in (("o", Hq), ("od", Hq), ("dq", Hq), ("dk", Hkv), ("dv", Hkv), ("dqd", Hq),
                 ("dkd", Hkv), ("dvd", Hkv)):
        out[k] = torch.full((N, H * D + 8), MARK, dtype=torch.bfloat16, device="cuda")[:, 8:]
    out["lse"], out["rbar"] = (torch.full((Hq, N), MARK, device="cuda") for _ in range(2))
    # a workspace full of NaN: nothing of it is read before it is written
    out["work"] = torch.full((native.mf_attn_window_work_bytes(N, Hq, Hkv, D, window, sinks, dual),), 255,
                             dtype=torch.uint8, device="cuda")
    out["status"] = torch.zeros(1, dtype=torch.int32, device="cuda")
    return out


def run(native, v, lens, Hq, Hkv, D, window, sinks, scale=0.0, starts=None, stream=None, out=None, n_seq=1):
    """Both passes on the GPU; returns the outputs (all rows)."""
    dual, N = "qd" in v, v["q"].shape[0]
    if out is None:
        out = buffers(native, N, Hq, Hkv, D, window, sinks, dual)
    t = lambda *names: {n: out[n] for n in names} if dual else {}
    if starts is None and lens is not None:
        starts = au.starts_of(lens).cuda()
    kw = dict(n_heads=Hq, n_kv_heads=Hkv, head_dim=D, window=window, n_sink=sinks, scale=scale,
              status=out["status"], stream=stream, seq_start=starts, n_seq=n_seq,
              **({k: v[k] for k in ("qd", "kd", "vd")} if dual else {}), **t("od", "rbar"))
    native.mf_attn_window_fwd(v["q"], v["k"], v["v"], out["o"], out["lse"], **kw)
    native.mf_attn_window_bwd(v["q"], v["k"], v["v"], out["o"], out["lse"], v["do"], out["dq"], out["dk"],
                              out["dv"], work=out["work"], dod=v.get("dod"), **t("dqd", "dkd", "dvd"), **kw)
    return out
