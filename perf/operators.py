"""What the speed of the attention operators is measured on: the calls that a training program
makes of them, on packed batches of token rows.

Two families of operators, each with its backward pass and with forward tangents (a tangent
rides along every value, so that forward-over-reverse products run through them):

* ``rope``  RMS norm of every query and key head (gains optional), then the rotary position of
  its token, from the rows of the fused q | k | v projection;
* ``attn``  causal attention with grouped key/value heads over packed sequences of different
  lengths.  ``fwd`` is the forward pass alone, ``train`` the forward and the backward pass.

With ``own`` false ``run`` computes them in elementary torch operations in float32, with
``own`` true through the calls of ``paper_2505_00793_gb300.native``.  A case is a dict of plain
values: ``listed()`` names twelve, ``draw(rng)`` makes one more of the same ranges.

Rows of a packed batch are tokens: sequence b owns rows seq_start[b] .. seq_start[b+1]-1, and
``tail`` rows follow the last sequence, which no call touches.
"""
from __future__ import annotations

import math
import random

import torch

own = False

F32, F64, BF16 = torch.float32, torch.float64, torch.bfloat16
DTYPES = {"f32": F32, "bf16": BF16}

# A float64 evaluation is given up to this many multiply-adds (a few seconds).
EXACT_OPS = 4e12


def _rope(name, way, n, heads, kv, dim, **kw):
    c = dict(name=name, kind="rope", way=way, n=n, seqs=4, pattern="ragged", lseed=1, tail=0,
             heads=heads, kv=kv, dim=dim, dual=False, norm=True, x="f32", y="bf16",
             layout="half", rot=0, base=10000.0, scaling="none", factor=1.0, orig=0,
             low=1.0, high=4.0, mscale=1.0, first=-1)
    c.update(kw)
    return c


def _attn(name, way, n, heads, kv, dim, **kw):
    c = dict(name=name, kind="attn", way=way, n=n, seqs=4, pattern="ragged", lseed=1, tail=0,
             heads=heads, kv=kv, dim=dim, dual=False)
    c.update(kw)
    return c


def listed():
    return [
        # One short document through the smallest heads: launches and their latency.
        _rope("rope_tiny_fwd", "fwd", 7, 2, 1, 16, seqs=2),
        # The larger transformer's layer (8 sequences of 1024, 16 heads of 64) in a step that
        # carries tangents: projections leave the GEMM as float32, operands of the attention
        # are bf16.
        _rope("rope_layer_dual_fwd", "fwd", 8192, 16, 16, 64, seqs=8, pattern="equal", dual=True),
        # Its backward pass with tangents, grouped heads, ragged documents: gradients of the
        # projection rows and of the gains.
        _rope("rope_layer_dual_bwd", "bwd", 8192, 16, 4, 64, seqs=11, tail=37, dual=True),
        # Rotary positions alone, on bf16 rows: half of each head in the interleaved order, far
        # positions (a window deep inside a long text) with a context scaled by frequency bands.
        _rope("rope_far_positions", "fwd", 40001, 8, 2, 128, norm=False, x="bf16",
              layout="interleaved", rot=64, base=500000.0, scaling="bands", factor=8.0,
              orig=8192, mscale=1.1, first=900000),
        # Rotary positions and norms in float32 for a float32 model, forward and backward.
        _rope("rope_fp32_bwd", "bwd", 5003, 12, 3, 80, seqs=9, y="f32", layout="interleaved",
              rot=40, scaling="base", factor=4.0),
        # A document of one token and one of 32: launches and their latency.
        _attn("attn_tiny_fwd", "fwd", 33, 4, 2, 32, seqs=2, pattern="one_first"),
        # The smaller transformer's batch (16 sequences of 256, 8 heads of 64): its inner step.
        _attn("attn_small_train", "train", 4096, 8, 8, 64, seqs=16, pattern="equal"),
        # A packed batch of ragged documents with grouped heads, one inner training step.
        _attn("attn_ragged_train", "train", 8192, 16, 4, 64, seqs=13, tail=51),
        # The larger transformer's layer with tangents: the forward half of a Hessian-vector
        # product.
        _attn("attn_layer_dual_fwd", "fwd", 8192, 16, 16, 64, seqs=8, pattern="equal", dual=True),
        # The whole Hessian-vector product's attention on ragged documents with grouped heads.
        _attn("attn_ragged_dual_train", "train", 8192, 16, 4, 64, seqs=10, dual=True),
        # One long document with wide heads that share one key/value head, forward only: an
        # evaluation of the outer loss.
        _attn("attn_long_fwd", "fwd", 16384, 8, 1, 128, seqs=1),
        # Long documents with wide heads, one training step: the largest case.
        _attn("attn_wide_train", "train", 12289, 16, 4, 128, seqs=3),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    heads, kv = rng.choice([(1, 1), (2, 1), (4, 4), (4, 2), (6, 3), (8, 8), (8, 1), (12, 4), (16, 4)])
    dual = rng.random() < 0.5
    common = dict(seqs=_log_int(rng, 1, 40), pattern=rng.choice(["ragged", "ragged", "equal", "one_first"]),
                  lseed=rng.randrange(1 << 30), tail=rng.choice([0, 0, 1, rng.randrange(1, 200)]), dual=dual)
    if rng.random() < 0.4:
        dim = 8 * rng.randrange(1, 17)
        norm = rng.random() < 0.7
        x, y = rng.choice([("f32", "bf16"), ("f32", "bf16"), ("bf16", "bf16"), ("f32", "f32")])
        c = _rope("", rng.choice(["fwd", "bwd"]), _log_int(rng, 1, 20000), heads, kv, dim,
                  norm=norm, x=x, y=y, layout=rng.choice(["half", "interleaved"]),
                  rot=rng.choice([0, 0, 2 * rng.randrange(1, dim // 2 + 1)]),
                  base=rng.choice([1e4, 5e5]), scaling=rng.choice(["none", "linear", "base", "bands"]),
                  factor=rng.choice([1.0, 2.0, 8.0]), orig=rng.choice([256, 8192]),
                  mscale=rng.choice([1.0, 1.1]), first=rng.choice([-1, -1, 0, 900000]), **common)
        if c["rot"] == 2 and c["scaling"] == "base":
            c["scaling"] = "linear"      # one pair turns at rate 1 whatever the base
        if not norm and x != y:
            c["x"] = y
    else:
        dim = 8 * rng.randrange(1, 9 if dual else 17)
        c = _attn("", rng.choice(["fwd", "train"]), _log_int(rng, 1, 6000), heads, kv, dim, **common)
    del c["name"]
    return c


def _lens(c):
    """Lengths of the packed sequences: equal ones, ragged ones (some may be empty), or ragged
    ones behind a sequence of one token."""
    n, k = c["n"], c["seqs"]
    if c["pattern"] == "equal":
        return [n // k + (1 if i < n % k else 0) for i in range(k)]
    r = random.Random(c["lseed"])
    cuts = sorted(r.randrange(n + 1) for _ in range(k - 1))
    if c["pattern"] == "one_first" and k > 1 and n > 1:
        cuts = [1] + [max(1, x) for x in cuts[1:]]
    return [b - a for a, b in zip([0] + cuts, cuts + [n])]


def _width(c):
    return (c["heads"] + 2 * c["kv"]) * c["dim"]


def prepare(case, seed):
    c = case
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    N, W, D = c["n"] + c["tail"], _width(c), c["dim"]

    def rnd(*shape, std=1.0, dtype=F32):
        return (torch.randn(*shape, device="cuda", generator=g) * std).to(dtype)

    lens = _lens(c)
    starts = [sum(lens[:i]) for i in range(len(lens) + 1)]
    s = {"case": c, "lens": lens,
         "seq_start": torch.tensor(starts, dtype=torch.int32, device="cuda"), "keep": {}}
    if c["kind"] == "rope":
        xt, yt = DTYPES[c["x"]], DTYPES[c["y"]]
        s["x"] = rnd(N, W, dtype=xt)
        s["xd"] = rnd(N, W, std=0.5, dtype=xt) if c["dual"] else None
        for k in ("gq", "gk"):
            s[k] = 1.0 + rnd(D, std=0.1) if c["norm"] else None
            s[k + "d"] = rnd(D, std=0.1) if c["norm"] and c["dual"] else None
        # positions: of the token in its sequence, or given for each row
        s["pos"] = None
        if c["first"] >= 0:
            s["pos"] = (torch.arange(N, device="cuda") + c["first"]).to(torch.int32)
        if c["way"] == "bwd":
            s["dy"] = rnd(N, W, dtype=yt)
            s["dyd"] = rnd(N, W, std=0.5, dtype=yt) if c["dual"] else None
        out = ["y"] if c["way"] == "fwd" else ["dx"]
        for k in out + [o + "d" for o in out] * c["dual"]:
            s[k] = torch.zeros(N, W, dtype=yt, device="cuda")
        if c["way"] == "bwd" and c["norm"]:
            for k in ["dgq", "dgk"] + ["dgqd", "dgkd"] * c["dual"]:
                s[k] = torch.zeros(D, device="cuda")
        return s
    Hq, Hkv = c["heads"], c["kv"]
    names = [""] + ["d"] * c["dual"]
    for t in names:
        # q, k and v are column ranges of one buffer of rows, as the rotary step leaves them
        x = rnd(N, W, std=0.5 if t else 1.0, dtype=BF16)
        s["q" + t], s["k" + t], s["v" + t] = x.split([Hq * D, Hkv * D, Hkv * D], 1)
        s["o" + t] = torch.zeros(N, Hq * D, dtype=BF16, device="cuda")
        s["rbar" if t else "lse"] = torch.zeros(Hq, N, device="cuda")
        if c["way"] == "train":
            s["do" + t] = rnd(N, Hq * D, std=0.5 if t else 1.0, dtype=BF16)
            dx = torch.zeros(N, W, dtype=BF16, device="cuda")
            s["dx" + t] = dx
            s["dq" + t], s["dk" + t], s["dv" + t] = dx.split([Hq * D, Hkv * D, Hkv * D], 1)
    # which row each place of a [sequences][longest] grid (or of one grid of all the rows,
    # where that is smaller) holds, and which pairs of places attend
    L, B, n = max(lens), len(lens), c["n"]
    if B * L * L > n * n:
        at = torch.arange(n, device="cuda").view(1, n)
        seq = torch.repeat_interleave(torch.arange(B, device="cuda"), torch.tensor(lens, device="cuda")).view(1, n)
        there = torch.ones(1, n, dtype=torch.bool, device="cuda")
    else:
        i = torch.arange(L, device="cuda").view(1, L)
        there = i < torch.tensor(lens, device="cuda").view(B, 1)
        at = torch.where(there, i + s["seq_start"][:-1].long().view(B, 1), 0)
        seq = torch.zeros(B, L, dtype=torch.long, device="cuda")
    i = torch.arange(at.shape[1], device="cuda")
    s["at"], s["there"] = at, there
    s["pairs"] = (i.view(1, -1, 1) >= i.view(1, 1, -1)) & (seq.unsqueeze(2) == seq.unsqueeze(1)) \
        & there.unsqueeze(2) & there.unsqueeze(1)
    return s


# ---- the plain forms ---------------------------------------------------------------------

def _turns(c, dtype, device):
    """Radians per position of each rotated pair."""
    R = c["rot"] or c["dim"]
    j = torch.arange(R // 2, dtype=dtype, device=device)
    base = c["base"]
    if c["scaling"] == "base":
        base = base * c["factor"] ** (R / (R - 2))
    w = base ** (-2.0 * j / R)
    if c["scaling"] == "linear":
        w = w / c["factor"]
    if c["scaling"] == "bands":
        turns = c["orig"] * w / (2 * math.pi)
        keep = ((turns - c["low"]) / (c["high"] - c["low"])).clamp(0, 1)
        w = w * (keep + (1 - keep) / c["factor"])
    return w


def _positions(s):
    c = s["case"]
    N = c["n"] + c["tail"]
    if s["pos"] is not None:
        return s["pos"].long(), N
    i = torch.arange(c["n"], device="cuda")
    seq = torch.searchsorted(s["seq_start"][1:].long(), i, right=True)
    return i - s["seq_start"].long()[seq], c["n"]


def _angles(s):
    """cos and sin [rows][1][pairs] in float32, from angles in 64 bits."""
    c = s["case"]
    pos, n = _positions(s)
    a = pos.to(F64).unsqueeze(1) * _turns(c, F64, "cuda")
    return (torch.cos(a) * c["mscale"]).to(F32).unsqueeze(1), (torch.sin(a) * c["mscale"]).to(F32).unsqueeze(1), n


def _rotate(c, z, cos, sin):
    R = c["rot"] or c["dim"]
    out = z.clone()
    if c["layout"] == "half":
        a, b = z[..., :R // 2], z[..., R // 2:R]
        out[..., :R // 2], out[..., R // 2:R] = a * cos - b * sin, b * cos + a * sin
    else:
        a, b = z[..., 0:R:2], z[..., 1:R:2]
        out[..., 0:R:2], out[..., 1:R:2] = a * cos - b * sin, b * cos + a * sin
    return out


def _heads(c, x, n):
    """Query heads, key heads and the value columns of the first n rows."""
    Hq, Hkv, D = c["heads"], c["kv"], c["dim"]
    q, k, v = x[:n].float().split([Hq * D, Hkv * D, Hkv * D], 1)
    return q.view(n, Hq, D), k.view(n, Hkv, D), v


EPS = 1e-6


def _norm_rope(c, x, xd, g, gd, cos, sin):
    if not c["norm"]:
        return _rotate(c, x, cos, sin), None if xd is None else _rotate(c, xd, cos, sin)
    r = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
    y = _rotate(c, x * r * g, cos, sin)
    if xd is None:
        return y, None
    rd = -r * r * r * (x * xd).mean(-1, keepdim=True)
    return y, _rotate(c, (xd * r + x * rd) * g + x * r * gd, cos, sin)


def _norm_rope_bwd(c, dy, dyd, x, xd, g, gd, cos, sin):
    """dx, dx', dg, dg' of the heads."""
    dy = _rotate(c, dy, cos, -sin)
    dyd = None if dyd is None else _rotate(c, dyd, cos, -sin)
    if not c["norm"]:
        return dy, dyd, None, None
    r = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
    a = dy * g
    m = (x * a).mean(-1, keepdim=True)
    dx = a * r - x * (r * r * r * m)
    dg = (dy * x * r).sum((0, 1))
    if dyd is None:
        return dx, None, dg, None
    r3 = r * r * r
    rd = -r3 * (x * xd).mean(-1, keepdim=True)
    ad = dyd * g + dy * gd
    md = (xd * a + x * ad).mean(-1, keepdim=True)
    dxd = rd * a + r * ad - x * (3 * r * r * rd * m + r3 * md) - xd * (r3 * m)
    return dx, dxd, dg, (dyd * x * r + dy * (xd * r + x * rd)).sum((0, 1))


def _plain_rope(s):
    c = s["case"]
    cos, sin, n = _angles(s)
    xq, xk, xv = _heads(c, s["x"], n)
    xqd, xkd, xvd = _heads(c, s["xd"], n) if c["dual"] else (None,) * 3

    def rows(like, q, k, v):
        out = torch.zeros_like(like)
        out[:n] = torch.cat([q.flatten(1), k.flatten(1), v], 1).to(like.dtype)
        return out

    if c["way"] == "fwd":
        q, qd = _norm_rope(c, xq, xqd, s["gq"], s["gqd"], cos, sin)
        k, kd = _norm_rope(c, xk, xkd, s["gk"], s["gkd"], cos, sin)
        out = {"y": rows(s["y"], q, k, xv)}
        if c["dual"]:
            out["yd"] = rows(s["yd"], qd, kd, xvd)
        return out
    dq, dk, dv = _heads(c, s["dy"], n)
    dqd, dkd, dvd = _heads(c, s["dyd"], n) if c["dual"] else (None,) * 3
    q, qd, gq, gqd = _norm_rope_bwd(c, dq, dqd, xq, xqd, s["gq"], s["gqd"], cos, sin)
    k, kd, gk, gkd = _norm_rope_bwd(c, dk, dkd, xk, xkd, s["gk"], s["gkd"], cos, sin)
    out = {"dx": rows(s["dx"], q, k, dv)}
    if c["norm"]:
        out.update(dgq=gq, dgk=gk)
    if c["dual"]:
        out["dxd"] = rows(s["dxd"], qd, kd, dvd)
        if c["norm"]:
            out.update(dgqd=gqd, dgkd=gkd)
    return out


def _grid(s, x, heads):
    """[grid][heads][places][dim] in float32 from rows."""
    c = s["case"]
    return x.float()[s["at"]].unflatten(2, (heads, c["dim"])).transpose(1, 2)


def _shared(c, x):
    return x.repeat_interleave(c["heads"] // c["kv"], 1)


def _summed(c, x):
    return x.unflatten(1, (c["kv"], c["heads"] // c["kv"])).sum(2)


def _ungrid(s, out, x):
    """Writes the places that hold a row to the rows of a new tensor like `out`."""
    out = torch.zeros_like(out)
    x = x.transpose(1, 2).flatten(2)[s["there"]].to(out.dtype)
    out[s["at"][s["there"]]] = x
    return out


def _plain_attn(s):
    c = s["case"]
    D, Hq, Hkv, N = c["dim"], c["heads"], c["kv"], c["n"] + c["tail"]
    scale = 1.0 / math.sqrt(D)
    q, k, v = _grid(s, s["q"], Hq), _shared(c, _grid(s, s["k"], Hkv)), _shared(c, _grid(s, s["v"], Hkv))
    pairs = s["pairs"].unsqueeze(1)
    S = (q @ k.transpose(-1, -2)).mul_(scale).masked_fill_(~pairs, -1e30)
    m = S.amax(-1, keepdim=True)
    P = S.sub_(m).exp_().mul_(pairs)
    l = P.sum(-1, keepdim=True).clamp_min_(1e-30)
    P = P.div_(l)
    o = P @ v
    lse = m + torch.log(l)
    out = {"o": _ungrid(s, s["o"], o)}

    def stat(x):
        z = torch.zeros(N, Hq, device="cuda")
        z[s["at"][s["there"]]] = x.squeeze(-1).transpose(1, 2)[s["there"]]
        return z.t().contiguous()

    out["lse"] = stat(lse)
    if c["dual"]:
        qd, kd = _grid(s, s["qd"], Hq), _shared(c, _grid(s, s["kd"], Hkv))
        vd = _shared(c, _grid(s, s["vd"], Hkv))
        Sd = (qd @ k.transpose(-1, -2)).add_(q @ kd.transpose(-1, -2)).mul_(scale)
        Pd = Sd.mul_(P)
        rbar = Pd.sum(-1, keepdim=True)
        Pd = Pd.sub_(P * rbar)
        out["od"] = _ungrid(s, s["od"], Pd @ v + P @ vd)
        out["rbar"] = stat(rbar)
    if c["way"] == "fwd":
        return out
    do = _grid(s, s["do"], Hq) * s["there"].view(*s["there"].shape[:1], 1, -1, 1)
    X = (do @ v.transpose(-1, -2))
    X = X.sub_((do * o).sum(-1, keepdim=True))
    dS = P * X
    dq, dk, dv = dS @ k, dS.transpose(-1, -2) @ q, P.transpose(-1, -2) @ do
    if c["dual"]:
        dod = _grid(s, s["dod"], Hq) * s["there"].view(*s["there"].shape[:1], 1, -1, 1)
        od = Pd @ v + P @ vd
        Xd = (dod @ v.transpose(-1, -2)).add_(do @ vd.transpose(-1, -2))
        Xd = Xd.sub_((dod * o + do * od).sum(-1, keepdim=True))
        dSd = Xd.mul_(P).add_(X.mul_(Pd))
        dqd = dSd @ k + dS @ kd
        dkd = dSd.transpose(-1, -2) @ q + dS.transpose(-1, -2) @ qd
        dvd = Pd.transpose(-1, -2) @ do + P.transpose(-1, -2) @ dod
        out["dqd"] = _ungrid(s, s["dqd"], dqd * scale)
        out["dkd"] = _ungrid(s, s["dkd"], _summed(c, dkd) * scale)
        out["dvd"] = _ungrid(s, s["dvd"], _summed(c, dvd))
    out["dq"] = _ungrid(s, s["dq"], dq * scale)
    out["dk"] = _ungrid(s, s["dk"], _summed(c, dk) * scale)
    out["dv"] = _ungrid(s, s["dv"], _summed(c, dv))
    return out


# ---- the framework's calls ---------------------------------------------------------------

def _own_rope(s):
    from paper_2505_00793_gb300 import native
    c, keep = s["case"], s["keep"]
    if not keep:
        keep["rope"] = native.rope_desc(layout=c["layout"], dims=c["rot"], base=c["base"],
                                        scaling=c["scaling"], factor=c["factor"],
                                        orig_len=c["orig"], low_turns=c["low"],
                                        high_turns=c["high"], mscale=c["mscale"])
        keep["work"] = torch.empty(native.mf_qk_rope_work_bytes(
            c["n"] + c["tail"], c["heads"], c["kv"], c["dim"], c["dual"]), dtype=torch.uint8, device="cuda")
    kw = dict(n_heads=c["heads"], n_kv_heads=c["kv"], head_dim=c["dim"], rope=keep["rope"],
              n_copy_heads=c["kv"], gq=s["gq"], gk=s["gk"], gqd=s["gqd"], gkd=s["gkd"], eps=EPS,
              pos=s["pos"], seq_start=s["seq_start"] if s["pos"] is None else None)
    if c["way"] == "fwd":
        native.mf_qk_rope_fwd(s["x"], s["y"], xd=s["xd"], yd=s.get("yd"), **kw)
        return {k: s[k] for k in ["y"] + ["yd"] * c["dual"]}
    names = ["dx"] + ["dxd"] * c["dual"] + (["dgq", "dgk"] + ["dgqd", "dgkd"] * c["dual"]) * c["norm"]
    native.mf_qk_rope_bwd(s["dy"], s["dx"], x=s["x"] if c["norm"] else None,
                          xd=s["xd"] if c["norm"] else None, dyd=s["dyd"], dxd=s.get("dxd"),
                          dgq=s.get("dgq"), dgk=s.get("dgk"), dgqd=s.get("dgqd"),
                          dgkd=s.get("dgkd"), work=keep["work"], **kw)
    return {k: s[k] for k in names}


def _own_attn(s):
    from paper_2505_00793_gb300 import native
    c, keep = s["case"], s["keep"]
    kw = dict(n_heads=c["heads"], n_kv_heads=c["kv"], head_dim=c["dim"], seq_start=s["seq_start"],
              qd=s.get("qd"), kd=s.get("kd"), vd=s.get("vd"), od=s.get("od"), rbar=s.get("rbar"))
    native.mf_attn_fwd(s["q"], s["k"], s["v"], s["o"], s["lse"], **kw)
    names = ["o", "lse"] + ["od", "rbar"] * c["dual"]
    if c["way"] == "train":
        if not keep:
            keep["work"] = torch.empty(native.mf_attn_work_bytes(c["n"] + c["tail"], c["heads"], c["dual"]),
                                       dtype=torch.uint8, device="cuda")
        native.mf_attn_bwd(s["q"], s["k"], s["v"], s["o"], s["lse"], s["do"], s["dq"], s["dk"],
                           s["dv"], dod=s.get("dod"), dqd=s.get("dqd"), dkd=s.get("dkd"),
                           dvd=s.get("dvd"), work=keep["work"], **kw)
        names += ["dq", "dk", "dv"] + ["dqd", "dkd", "dvd"] * c["dual"]
    return {k: s[k] for k in names}


def run(state):
    rope = state["case"]["kind"] == "rope"
    if own:
        return _own_rope(state) if rope else _own_attn(state)
    return _plain_rope(state) if rope else _plain_attn(state)


# ---- what a pass cannot do without ---------------------------------------------------------

def work(case):
    c = case
    n, W, D = c["n"], _width(c), c["dim"]
    two = 2 if c["dual"] else 1
    if c["kind"] == "rope":
        if c["first"] >= 0:
            n += c["tail"]
        xb, yb = (4 if c["x"] == "f32" else 2), (4 if c["y"] == "f32" else 2)
        qk = (c["heads"] + c["kv"]) * D
        if c["way"] == "fwd":
            per = W * (xb + yb)
        else:   # gradients in and out, and the q and k columns of the rows for the norm
            per = W * 2 * yb + (qk * xb if c["norm"] else 0)
        return {"bytes": float(n * per * two + (4 * n if c["first"] >= 0 else 0)),
                "flops": float(n * qk * two * ((12 if c["norm"] else 4) * (1 if c["way"] == "fwd" else 2)))}
    # float64-exact integers: pairs of a query and a key it attends to, over the heads
    pairs = sum(x * (x + 1) // 2 for x in _lens(c)) * c["heads"]
    prod = 2 * D * pairs
    rows = n * W * 2 + n * c["heads"] * D * 2
    stats = n * c["heads"] * 4
    b, f = (rows + stats) * two, 2 * prod * (3 if c["dual"] else 1)
    if c["way"] == "train":
        b += (n * c["heads"] * D * 2 + n * W * 2) * two
        f += 4 * prod * (3 if c["dual"] else 1)
    return {"bytes": float(b), "flops": float(f)}


# ---- float64 from the definitions ----------------------------------------------------------

def _exact_rope(s):
    c = s["case"]
    Hq, Hkv, D = c["heads"], c["kv"], c["dim"]
    N = c["n"] + c["tail"]
    R = c["rot"] or D
    rows = N if c["first"] >= 0 else c["n"]
    if c["first"] >= 0:
        pos = torch.arange(N, dtype=F64, device="cuda") + c["first"]
    else:
        pos = torch.cat([torch.arange(x, dtype=F64, device="cuda") for x in _lens(c)])
    # one complex rotation factor per pair, frequency by frequency
    fac = []
    for j in range(R // 2):
        base = c["base"] * (c["factor"] ** (R / (R - 2)) if c["scaling"] == "base" else 1.0)
        w = math.pow(base, -2.0 * j / R)
        if c["scaling"] == "linear":
            w /= c["factor"]
        elif c["scaling"] == "bands":
            t = c["orig"] / (2 * math.pi / w)
            if t < c["low"]:
                w /= c["factor"]
            elif t <= c["high"]:
                f = (t - c["low"]) / (c["high"] - c["low"])
                w = (1 - f) * w / c["factor"] + f * w
        fac.append(torch.polar(torch.full_like(pos, c["mscale"]), pos * w))
    fac = torch.stack(fac, 1).unsqueeze(1)

    def head(x, g):
        x = x.unflatten(1, (-1, D))
        if c["norm"]:
            x = x / torch.sqrt(x.square().sum(-1, keepdim=True) / D + EPS) * g
        z = x[..., :R]
        z = torch.complex(z[..., :R // 2], z[..., R // 2:]) if c["layout"] == "half" else \
            torch.view_as_complex(z.reshape(*z.shape[:-1], R // 2, 2).contiguous())
        z = z * fac
        z = torch.cat([z.real, z.imag], -1) if c["layout"] == "half" else torch.view_as_real(z).flatten(-2)
        return torch.cat([z, x[..., R:]], -1).flatten(1)

    def f(x, gq, gk):
        q, k, v = x.split([Hq * D, Hkv * D, Hkv * D], 1)
        return torch.cat([head(q, gq), head(k, gk), v], 1)

    one = torch.ones(D, dtype=F64, device="cuda")
    prim = (s["x"][:rows].double(),) + tuple(one if s[k] is None else s[k].double() for k in ("gq", "gk"))
    tang = (s["xd"][:rows].double(),) + tuple(0 * one if s[k] is None else s[k].double() for k in ("gqd", "gkd")) \
        if c["dual"] else None

    def whole(x):
        out = torch.zeros(N, x.shape[1], dtype=F64, device="cuda")
        out[:rows] = x
        return out

    if c["way"] == "fwd":
        if not c["dual"]:
            return {"y": whole(f(*prim))}
        y, yd = torch.func.jvp(f, prim, tang)
        return {"y": whole(y), "yd": whole(yd)}

    def grads(x, gq, gk, dy):
        return torch.func.vjp(f, x, gq, gk)[1](dy)

    dy = s["dy"][:rows].double()
    if c["dual"]:
        g, gd = torch.func.jvp(grads, prim + (dy,), tang + (s["dyd"][:rows].double(),))
    else:
        g, gd = grads(*prim, dy), None
    out = {"dx": whole(g[0])}
    if c["norm"]:
        out.update(dgq=g[1], dgk=g[2])
    if gd is not None:
        out["dxd"] = whole(gd[0])
        if c["norm"]:
            out.update(dgqd=gd[1], dgkd=gd[2])
    return out


def _exact_attn(s):
    c = s["case"]
    Hq, Hkv, D = c["heads"], c["kv"], c["dim"]
    N = c["n"] + c["tail"]
    out = {"o": torch.zeros(N, Hq * D, dtype=F64, device="cuda"),
           "lse": torch.zeros(Hq, N, dtype=F64, device="cuda")}
    if c["dual"]:
        out.update(od=torch.zeros_like(out["o"]), rbar=torch.zeros_like(out["lse"]))
    train = c["way"] == "train"
    for t in [""] + ["d"] * c["dual"]:
        if train:
            for k, h in (("dq", Hq), ("dk", Hkv), ("dv", Hkv)):
                out[k + t] = torch.zeros(N, h * D, dtype=F64, device="cuda")
    a = 0
    for L in _lens(c):
        r, a = slice(a, a + L), a + L
        if not L:
            continue
        later = torch.ones(L, L, dtype=torch.bool, device="cuda").triu(1)
        for h in range(Hkv):     # one group of query heads and its key/value head at a time
            G = Hq // Hkv
            qc, kc = slice(h * G * D, (h + 1) * G * D), slice(h * D, (h + 1) * D)

            def part(name, cols):
                return s[name][r, cols].double()

            def f(q, k, v):
                z = torch.einsum("igd,jd->gij", q.unflatten(1, (G, D)), k) * D ** -0.5
                z = z.masked_fill(later, -math.inf)
                lse = torch.logsumexp(z, -1)
                return torch.einsum("gij,jd->igd", torch.exp(z - lse.unsqueeze(-1)), v).flatten(1), lse

            def grads(q, k, v, do):
                return torch.func.vjp(lambda *x: f(*x)[0], q, k, v)[1](do)

            prim = (part("q", qc), part("k", kc), part("v", kc))
            heads = slice(h * G, (h + 1) * G)
            if c["dual"]:
                tang = (part("qd", qc), part("kd", kc), part("vd", kc))
                (o, lse), (od, rbar) = torch.func.jvp(f, prim, tang)
                out["od"][r, qc], out["rbar"][heads, r] = od, rbar
            else:
                o, lse = f(*prim)
            out["o"][r, qc], out["lse"][heads, r] = o, lse
            if not train:
                continue
            if c["dual"]:
                g, gd = torch.func.jvp(grads, prim + (part("do", qc),), tang + (part("dod", qc),))
            else:
                g, gd = grads(*prim, part("do", qc)), None
            for i, (k, cols) in enumerate((("dq", qc), ("dk", kc), ("dv", kc))):
                out[k][r, cols] = g[i]
                if gd is not None:
                    out[k + "d"][r, cols] = gd[i]
    return out


def exact(case, seed):
    c = case
    if c["kind"] == "attn":
        ops = sum(x * x for x in _lens(c)) * c["heads"] * c["dim"] * 2
        if ops * (4 if c["dual"] else 1) * (3 if c["way"] == "train" else 1) > EXACT_OPS:
            return None
    s = prepare(case, seed)
    return _exact_rope(s) if c["kind"] == "rope" else _exact_attn(s)
