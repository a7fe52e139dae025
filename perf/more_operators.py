"""What the speed of two more operators on packed token rows is measured on: the calls that a
training program makes of them.

* ``embed``   rows of an embedding table by token id, scaled (``fwd``), and the gradient of the
  table (``bwd``): every row of it the sum over the tokens that have its id;
* ``window``  causal attention with grouped key/value heads over packed sequences in which a row
  attends to itself, the ``window - 1`` rows before it and the first ``sinks`` rows of its sequence.
  ``fwd`` is the forward pass alone, ``train`` the forward and the backward pass.

Both with forward tangents (``dual``: a tangent rides along every value, so that
forward-over-reverse products run through them).  With ``own`` false ``run`` computes them in
elementary torch operations in float32, with ``own`` true through the calls of
``paper_2505_00793_gb300.native``.  A case is a dict of plain values: ``listed()`` names twelve,
``draw(rng)`` makes one more of the same ranges.

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


def _embed(name, way, n, vocab, dim, **kw):
    c = dict(name=name, kind="embed", way=way, n=n, vocab=vocab, dim=dim, seqs=1, pattern="equal", lseed=1,
             tail=0, ids="zipf", pad=0.0, dual=False, e="f32", y="f32", scale=1.0)
    c.update(kw)
    return c


def _window(name, way, n, heads, kv, dim, window, sinks, **kw):
    c = dict(name=name, kind="window", way=way, n=n, heads=heads, kv=kv, dim=dim, window=window, sinks=sinks,
             seqs=4, pattern="ragged", lseed=1, tail=0, dual=False)
    c.update(kw)
    return c


def listed():
    return [
        # A few tokens through the smallest table: launches and their latency.
        _embed("embed_tiny_fwd", "fwd", 7, 50, 16, scale=4.0),
        # The larger transformer's batch (8 sequences of 1024, 32768 ids, width 1024) in a step
        # that carries tangents: float32 parameters and residual rows.
        _embed("embed_layer_dual_fwd", "fwd", 8192, 32768, 1024, dual=True, scale=32.0),
        # Its gradient with tangents: most of a table's rows occur in no batch and are zeros.
        _embed("embed_layer_dual_bwd", "bwd", 8192, 32768, 1024, dual=True, scale=32.0),
        # The smaller transformer's batch (16 sequences of 256, 8192 ids, width 512), bf16 rows,
        # ragged documents with rows behind the last.
        _embed("embed_small_bwd", "bwd", 4096, 8192, 512, seqs=16, pattern="ragged", tail=19, y="bf16"),
        # A long packed batch of which three tenths are one id (a separator) and a tenth are rows
        # without a token, an odd table.
        _embed("embed_long_bwd", "bwd", 131071, 50001, 768, seqs=40, pattern="ragged", ids="one", pad=0.1,
               y="bf16", scale=27.7),
        # A document of one token and one of 32: launches and their latency.
        _window("window_tiny_fwd", "fwd", 33, 4, 2, 32, 8, 1, seqs=2, pattern="one_first"),
        # The smaller transformer's batch with a short window: its inner step.
        _window("window_small_train", "train", 4096, 8, 8, 64, 64, 4, seqs=16, pattern="equal"),
        # Sequences of the larger transformer's length, a window of one tile, no sinks.
        _window("window_short_fwd", "fwd", 16384, 16, 8, 64, 128, 0, seqs=16, pattern="equal"),
        # One long document with grouped heads: an evaluation of the outer loss.
        _window("window_long_fwd", "fwd", 32768, 16, 4, 64, 1024, 4, seqs=1),
        # A packed batch of ragged documents, one inner training step.
        _window("window_ragged_train", "train", 16384, 16, 4, 64, 512, 4, seqs=13, tail=51),
        # The whole Hessian-vector product's attention, a window that ends inside tiles.
        _window("window_ragged_dual_train", "train", 8192, 16, 4, 64, 257, 1, seqs=6, dual=True),
        # Long documents with wide heads, one training step: the largest case.
        _window("window_wide_train", "train", 24577, 16, 2, 128, 1000, 16, seqs=3),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    common = dict(seqs=_log_int(rng, 1, 40), pattern=rng.choice(["ragged", "ragged", "equal", "one_first"]),
                  lseed=rng.randrange(1 << 30), tail=rng.choice([0, 0, 1, rng.randrange(1, 200)]),
                  dual=rng.random() < 0.5)
    if rng.random() < 0.4:
        dim = rng.choice([8 * _log_int(rng, 1, 256), _log_int(rng, 1, 1500)])
        n = _log_int(rng, 1, 100000)
        vocab = _log_int(rng, 1, 130000)
        while (n + vocab) * dim > 120e6:
            n, vocab = n // 2 + 1, vocab // 2 + 1
        c = _embed("", rng.choice(["fwd", "bwd", "bwd"]), n, vocab, dim,
                   ids=rng.choice(["zipf", "zipf", "uniform", "one"]), pad=rng.choice([0.0, 0.0, 0.1]),
                   e=rng.choice(["f32", "bf16"]), y=rng.choice(["f32", "bf16"]),
                   scale=rng.choice([1.0, math.sqrt(dim), 0.3]), **common)
    else:
        heads, kv = rng.choice([(1, 1), (2, 1), (4, 4), (4, 2), (6, 3), (8, 8), (8, 1), (12, 4), (16, 4)])
        dim = 8 * rng.randrange(1, 9 if common["dual"] else 17)
        n = _log_int(rng, 1, 16000)
        c = _window("", rng.choice(["fwd", "train"]), n, heads, kv, dim, _log_int(rng, 1, 4000),
                    rng.choice([0, 1, 4, rng.randrange(0, 129)]), **common)
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


def _ld(cols):
    """Columns of a row buffer whose rows begin on 16-byte boundaries."""
    return -(-cols // 8) * 8


def prepare(case, seed):
    c = case
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    N, D = c["n"] + c["tail"], c["dim"]

    def rnd(rows, cols, std=1.0, dtype=F32):
        return (torch.randn(rows, _ld(cols), device="cuda", generator=g) * std).to(dtype)[:, :cols]

    def zeros(rows, cols, dtype=F32):
        return torch.zeros(rows, _ld(cols), dtype=dtype, device="cuda")[:, :cols]

    lens = _lens(c)
    starts = [sum(lens[:i]) for i in range(len(lens) + 1)]
    s = {"case": c, "lens": lens, "starts": starts,
         "seq_start": torch.tensor(starts, dtype=torch.int32, device="cuda"), "keep": {}}
    tangents = [""] + ["d"] * c["dual"]
    if c["kind"] == "embed":
        V, yt = c["vocab"], DTYPES[c["y"]]
        u = torch.rand(N, device="cuda", generator=g, dtype=F64)
        if c["ids"] == "uniform":
            ids = (u * V).long()
        else:      # the id of rank v with probability near 1 / (v + 1)
            ids = (torch.exp(u * math.log(V + 1.0)) - 1).long()
        ids = ids.clamp(0, V - 1)
        if c["ids"] == "one":
            ids[torch.rand(N, device="cuda", generator=g) < 0.3] = V // 2
        if c["pad"]:
            ids[torch.rand(N, device="cuda", generator=g) < c["pad"]] = -1
        s["ids"] = ids.to(torch.int32)
        for t in tangents:
            if c["way"] == "fwd":
                s["E" + t] = rnd(V, D, 0.5 if t else 1.0, DTYPES[c["e"]])
                s["y" + t] = zeros(N, D, yt)
            else:
                s["dy" + t] = rnd(N, D, 0.5 if t else 1.0, yt)
                s["dE" + t] = zeros(V, D)
        return s
    Hq, Hkv = c["heads"], c["kv"]
    cols = [Hq * D, Hkv * D, Hkv * D]
    for t in tangents:
        # q, k and v are column ranges of one buffer of rows, as the rotary step leaves them
        s["q" + t], s["k" + t], s["v" + t] = rnd(N, sum(cols), 0.5 if t else 1.0, BF16).split(cols, 1)
        s["o" + t] = zeros(N, Hq * D, BF16)
        s["rbar" if t else "lse"] = torch.zeros(Hq, N, device="cuda")
        if c["way"] == "train":
            s["do" + t] = rnd(N, Hq * D, 0.5 if t else 1.0, BF16)
            s["dq" + t], s["dk" + t], s["dv" + t] = zeros(N, sum(cols), BF16).split(cols, 1)
    return s


# ---- the plain forms ---------------------------------------------------------------------

def _plain_embed(s):
    c = s["case"]
    n, out = c["n"], {}
    ids = s["ids"][:n].long()
    real = (ids >= 0).unsqueeze(1)
    for t in [""] + ["d"] * c["dual"]:
        if c["way"] == "fwd":
            y = torch.zeros_like(s["y" + t])
            y[:n] = (s["E" + t][ids.clamp_min(0)].float() * c["scale"] * real).to(y.dtype)
            out["y" + t] = y
        else:
            dE = torch.zeros_like(s["dE" + t])
            dE.index_add_(0, ids.clamp_min(0), s["dy" + t][:n].float() * real)
            out["dE" + t] = dE.mul_(c["scale"])
    return out


# Query rows of a block of the plain form.
BLOCK = 512


def _blocks(s, size):
    """(query rows, key rows, which pairs attend) of every block of query rows; the keys are a
    sequence's sinks in front of the block's window, and the window."""
    c = s["case"]
    W, S = c["window"], c["sinks"]
    for lo, L in zip(s["starts"], s["lens"]):
        for a in range(lo, lo + L, size):
            b = min(a + size, lo + L)
            w = max(lo, a - W + 1)
            keys = torch.cat([torch.arange(lo, min(lo + S, w), device="cuda"), torch.arange(w, b, device="cuda")])
            i, j = torch.arange(a, b, device="cuda").unsqueeze(1), keys.unsqueeze(0)
            yield slice(a, b), keys, (j <= i) & ((i - j < W) | (j - lo < S))


def _heads(c, x, h):
    """[h][rows][dim] in float32 from rows of h heads."""
    return x.float().unflatten(1, (h, c["dim"])).transpose(0, 1)


def _rows(x):
    return x.transpose(0, 1).flatten(1)


def _plain_window(s):
    c = s["case"]
    D, Hq, Hkv = c["dim"], c["heads"], c["kv"]
    G, scale, train = Hq // Hkv, 1.0 / math.sqrt(c["dim"]), c["way"] == "train"
    out = {k: torch.zeros_like(s[k]) for k in ["o", "lse"] + ["od", "rbar"] * c["dual"]}
    acc = {}
    if train:
        for t in [""] + ["d"] * c["dual"]:
            out["dq" + t] = torch.zeros_like(s["dq" + t])
            for k in ("dk", "dv"):
                acc[k + t] = torch.zeros(s["k"].shape[0], Hkv * D, device="cuda")

    def grouped(x):
        """The keys' heads, each for its group's query heads."""
        return _heads(c, x, Hkv).repeat_interleave(G, 0)

    def summed(x):
        return _rows(x.unflatten(0, (Hkv, G)).sum(1))

    for r, keys, pairs in _blocks(s, BLOCK):
        q, k, v = _heads(c, s["q"][r], Hq), grouped(s["k"][keys]), grouped(s["v"][keys])
        S = (q @ k.mT).mul_(scale).masked_fill_(~pairs, -1e30)
        m = S.amax(-1, keepdim=True)
        P = S.sub_(m).exp_().mul_(pairs)
        l = P.sum(-1, keepdim=True)
        P = P.div_(l)
        o = P @ v
        out["o"][r] = _rows(o).to(BF16)
        out["lse"][:, r] = (m + torch.log(l)).squeeze(-1)
        if c["dual"]:
            qd, kd, vd = _heads(c, s["qd"][r], Hq), grouped(s["kd"][keys]), grouped(s["vd"][keys])
            Pd = (qd @ k.mT).add_(q @ kd.mT).mul_(scale).mul_(P)
            rbar = Pd.sum(-1, keepdim=True)
            Pd = Pd.sub_(P * rbar)
            od = Pd @ v + P @ vd
            out["od"][r] = _rows(od).to(BF16)
            out["rbar"][:, r] = rbar.squeeze(-1)
        if not train:
            continue
        do = _heads(c, s["do"][r], Hq)
        X = (do @ v.mT).sub_((do * o).sum(-1, keepdim=True))
        dS = P * X
        out["dq"][r] = _rows((dS @ k).mul_(scale)).to(BF16)
        acc["dk"].index_add_(0, keys, summed(dS.mT @ q))
        acc["dv"].index_add_(0, keys, summed(P.mT @ do))
        if c["dual"]:
            dod = _heads(c, s["dod"][r], Hq)
            Xd = (dod @ v.mT).add_(do @ vd.mT).sub_((dod * o + do * od).sum(-1, keepdim=True))
            dSd = Xd.mul_(P).add_(X.mul_(Pd))
            out["dqd"][r] = _rows((dSd @ k + dS @ kd).mul_(scale)).to(BF16)
            acc["dkd"].index_add_(0, keys, summed(dSd.mT @ q + dS.mT @ qd))
            acc["dvd"].index_add_(0, keys, summed(Pd.mT @ do + P.mT @ dod))
    for k, x in acc.items():
        out[k] = (x * scale if k.startswith("dk") else x).to(BF16)
    return out


# ---- the framework's calls ---------------------------------------------------------------

def _own_embed(s):
    from paper_2505_00793_gb300 import native
    c, keep = s["case"], s["keep"]
    if c["way"] == "fwd":
        native.mf_embed_fwd(s["ids"], s["E"], s["y"], scale=c["scale"], Ed=s.get("Ed"), yd=s.get("yd"),
                            seq_start=s["seq_start"])
        return {k: s[k] for k in ["y"] + ["yd"] * c["dual"]}
    if not keep:
        keep["work"] = torch.empty(native.mf_embed_work_bytes(c["n"] + c["tail"], c["vocab"], c["dim"], c["dual"]),
                                   dtype=torch.uint8, device="cuda")
    native.mf_embed_bwd(s["ids"], s["dy"], s["dE"], keep["work"], scale=c["scale"], dyd=s.get("dyd"),
                        dEd=s.get("dEd"), seq_start=s["seq_start"])
    return {k: s[k] for k in ["dE"] + ["dEd"] * c["dual"]}


def _own_window(s):
    from paper_2505_00793_gb300 import native
    c, keep = s["case"], s["keep"]
    kw = dict(n_heads=c["heads"], n_kv_heads=c["kv"], head_dim=c["dim"], window=c["window"], n_sink=c["sinks"],
              seq_start=s["seq_start"], qd=s.get("qd"), kd=s.get("kd"), vd=s.get("vd"), od=s.get("od"),
              rbar=s.get("rbar"))
    native.mf_attn_window_fwd(s["q"], s["k"], s["v"], s["o"], s["lse"], **kw)
    names = ["o", "lse"] + ["od", "rbar"] * c["dual"]
    if c["way"] == "train":
        if not keep:
            keep["work"] = torch.empty(native.mf_attn_window_work_bytes(
                c["n"] + c["tail"], c["heads"], c["kv"], c["dim"], c["window"], c["sinks"], c["dual"]),
                dtype=torch.uint8, device="cuda")
        native.mf_attn_window_bwd(s["q"], s["k"], s["v"], s["o"], s["lse"], s["do"], s["dq"], s["dk"],
                                  s["dv"], dod=s.get("dod"), dqd=s.get("dqd"), dkd=s.get("dkd"),
                                  dvd=s.get("dvd"), work=keep["work"], **kw)
        names += ["dq", "dk", "dv"] + ["dqd", "dkd", "dvd"] * c["dual"]
    return {k: s[k] for k in names}


def run(state):
    embed = state["case"]["kind"] == "embed"
    if own:
        return _own_embed(state) if embed else _own_window(state)
    return _plain_embed(state) if embed else _plain_window(state)


# ---- what a pass cannot do without ---------------------------------------------------------

def _distinct(c):
    """Rows of the table that a batch's tokens are expected to name."""
    V, n = c["vocab"], c["n"] * (1 - c["pad"]) * (0.7 if c["ids"] == "one" else 1.0)
    if c["ids"] == "uniform":
        p = torch.full((V,), 1.0 / V, dtype=F64)
    else:
        p = torch.log1p(1 / torch.arange(1, V + 1, dtype=F64)) / math.log(V + 1.0)
    return float((-torch.expm1(n * torch.log1p(-p.clamp_max(1 - 1e-12)))).sum())


def work(case):
    c = case
    n, D = c["n"], c["dim"]
    two = 2 if c["dual"] else 1
    if c["kind"] == "embed":
        row = n * D * (4 if c["y"] == "f32" else 2)
        table = _distinct(c) * D * (4 if c["e"] == "f32" else 2) if c["way"] == "fwd" else c["vocab"] * D * 4
        return {"bytes": float((row + table) * two + 4 * n), "flops": float(n * D * two)}
    Hq, Hkv, W, S = c["heads"], c["kv"], c["window"], c["sinks"]
    # pairs of a query and a key it attends to, over the heads: min(i + 1, W) in the window, and
    # the sinks in front of it
    pairs = 0
    for L in _lens(c):
        i = torch.arange(L, dtype=torch.int64)
        pairs += int(((i + 1).clamp_max(W) + (i + 1 - W).clamp(0, S)).sum())
    prod = 2 * D * pairs * Hq
    rows = n * (Hq + 2 * Hkv) * D * 2
    b, f = (rows + n * Hq * D * 2 + n * Hq * 4) * two, 2 * prod * (3 if c["dual"] else 1)
    if c["way"] == "train":
        b += (n * Hq * D * 2 + rows) * two
        f += 4 * prod * (3 if c["dual"] else 1)
    return {"bytes": float(b), "flops": float(f)}


# ---- float64 from the definitions ----------------------------------------------------------

def _exact_embed(s):
    c = s["case"]
    n, V = c["n"], c["vocab"]
    ids = s["ids"][:n].cpu()
    at = torch.nonzero(ids >= 0).squeeze(1)
    order = torch.argsort(ids[at], stable=True)
    at, which = at[order].cuda(), ids[at][order].long().cuda()
    out = {}
    for t in [""] + ["d"] * c["dual"]:
        if c["way"] == "fwd":
            y = torch.zeros(s["y" + t].shape, dtype=F64, device="cuda")
            y[at] = s["E" + t].double()[which] * c["scale"]
            out["y" + t] = y
            continue
        # sums of runs of equal ids, as differences of a running sum within blocks of columns
        dE = torch.zeros(V, c["dim"], dtype=F64, device="cuda")
        if len(at):
            names, counts = torch.unique_consecutive(which, return_counts=True)
            last = torch.cumsum(counts, 0) - 1
            for j in range(0, c["dim"], 64):
                run = torch.cumsum(s["dy" + t][at, j:j + 64].double(), 0)[last]
                dE[names, j:j + 64] = torch.diff(run, dim=0, prepend=torch.zeros_like(run[:1]))
        out["dE" + t] = dE * c["scale"]
    return out


def _exact_window(s):
    c = s["case"]
    Hq, Hkv, D = c["heads"], c["kv"], c["dim"]
    G, N, train = Hq // Hkv, c["n"] + c["tail"], c["way"] == "train"
    z = lambda h: torch.zeros(N, h * D, dtype=F64, device="cuda")
    out = {"o": z(Hq), "lse": torch.zeros(Hq, N, dtype=F64, device="cuda")}
    if c["dual"]:
        out.update(od=z(Hq), rbar=torch.zeros_like(out["lse"]))
    if train:
        for t in [""] + ["d"] * c["dual"]:
            out.update({"dq" + t: z(Hq), "dk" + t: z(Hkv), "dv" + t: z(Hkv)})
    for lo, L in zip(s["starts"], s["lens"]):
        for a in range(0, L, 1024):
            rows = torch.arange(a, min(a + 1024, L), device="cuda")
            first = max(0, a - c["window"] + 1)
            near = torch.arange(first, int(rows[-1]) + 1, device="cuda")
            far = torch.arange(0, min(c["sinks"], first), device="cuda")
            cols = torch.cat([far, near])
            age = rows.view(-1, 1) - cols.view(1, -1)
            away = (age < 0) | ((age >= c["window"]) & (cols >= c["sinks"]).view(1, -1))
            rows, cols = rows + lo, cols + lo
            for h in range(Hkv):     # one group of query heads and its key/value head at a time
                qc, kc = slice(h * G * D, (h + 1) * G * D), slice(h * D, (h + 1) * D)

                def part(name):
                    return s[name][rows, qc].double() if name[0] == "q" or name[:2] == "do" else \
                        s[name][cols, kc].double()

                def f(q, k, v):
                    e = torch.einsum("igd,jd->gij", q.unflatten(1, (G, D)), k) * D ** -0.5
                    e = e.masked_fill(away, -math.inf)
                    lse = torch.logsumexp(e, -1)
                    return torch.einsum("gij,jd->igd", torch.exp(e - lse.unsqueeze(-1)), v).flatten(1), lse

                def grads(q, k, v, do):
                    return torch.func.vjp(lambda *x: f(*x)[0], q, k, v)[1](do)

                prim = (part("q"), part("k"), part("v"))
                heads = slice(h * G, (h + 1) * G)
                if c["dual"]:
                    tang = (part("qd"), part("kd"), part("vd"))
                    (o, lse), (od, rbar) = torch.func.jvp(f, prim, tang)
                    out["od"][rows, qc], out["rbar"][heads, rows] = od, rbar
                else:
                    o, lse = f(*prim)
                out["o"][rows, qc], out["lse"][heads, rows] = o, lse
                if not train:
                    continue
                if c["dual"]:
                    g, gd = torch.func.jvp(grads, prim + (part("do"),), tang + (part("dod"),))
                else:
                    g, gd = grads(*prim, part("do")), None
                for t, x in (("", g), ("d", gd)):
                    if x is not None:
                        out["dq" + t][rows, qc] = x[0]
                        out["dk" + t][cols, kc] += x[1]
                        out["dv" + t][cols, kc] += x[2]
    return out


def exact(case, seed):
    c = case
    if c["kind"] == "window":
        ops = sum(x * min(x, c["window"] + 1024 + c["sinks"]) for x in _lens(c)) * c["heads"] * c["dim"] * 2
        if ops * (4 if c["dual"] else 1) * (3 if c["way"] == "train" else 1) > EXACT_OPS:
            return None
    s = prepare(case, seed)
    return _exact_embed(s) if c["kind"] == "embed" else _exact_window(s)
