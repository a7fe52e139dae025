"""The operators on packed token rows as a layer at the bottom of a decoder calls them, with one list of
sequences for all: ids through the embedding, projected rows through norms and rotary positions, attention
with a window and sinks, and all the way back to the table and the gains, with tangents; eager, and
captured and replayed with other tokens and lengths."""
import pytest

import attn_ops_util as au
from gpu_util import need_gpu

HQ, HKV, D, V, WINDOW, SINKS, SCALE = 4, 2, 64, 300, 50, 3, 2.0
COLS = [HQ * D, HKV * D, HKV * D]
W = sum(COLS)


def _tokens(torch, lens, N, seed):
    g = torch.Generator().manual_seed(seed)
    ids = torch.randint(0, V, (N,), generator=g, dtype=torch.int32)
    ids[torch.rand(N, generator=g) < 0.3] = 7                        # one frequent id
    ids[torch.rand(N, generator=g) < 0.05] = -1                      # padding
    do, dod = (torch.randn(N, HQ * D, generator=g) * s for s in (1.0, 0.5))
    return ids, do.bfloat16(), dod.bfloat16()


def _weights(torch, seed):
    g = torch.Generator().manual_seed(seed)
    rnd = lambda *s, std=1.0: torch.randn(*s, generator=g) * std
    return dict(E=rnd(V, W), Ed=rnd(V, W, std=0.5), gq=1 + rnd(D, std=0.2), gk=1 + rnd(D, std=0.2),
                gqd=rnd(D, std=0.2), gkd=rnd(D, std=0.2))


def _buffers(torch, native, N):
    f32, bf = (dict(dtype=t, device="cuda") for t in (torch.float32, torch.bfloat16))
    b = {}
    for t in ("", "d"):
        b["x" + t] = torch.empty(N, W, **f32)
        b["y" + t], b["dy" + t], b["dx" + t] = (torch.empty(N, W, **bf) for _ in range(3))
        b["o" + t] = torch.empty(N, HQ * D, **bf)
        b["dE" + t] = torch.empty(V, W, **f32)
        b["dgq" + t], b["dgk" + t] = (torch.empty(D, **f32) for _ in range(2))
    b["lse"], b["rbar"] = (torch.empty(HQ, N, **f32) for _ in range(2))
    byte = lambda n: torch.empty(n, dtype=torch.uint8, device="cuda")
    b["work"] = (byte(native.mf_attn_window_work_bytes(N, HQ, HKV, D, WINDOW, SINKS, True)),
                 byte(native.mf_qk_rope_work_bytes(N, HQ, HKV, D, True)), byte(native.mf_embed_work_bytes(N, V, W, True)))
    return b


def _run(native, w, ids, do, dod, starts, b):
    native.mf_embed_fwd(ids, w["E"], b["x"], scale=SCALE, Ed=w["Ed"], yd=b["xd"], seq_start=starts)
    rk = dict(n_heads=HQ, n_kv_heads=HKV, head_dim=D, rope=native.rope_desc(), n_copy_heads=HKV, gq=w["gq"], gk=w["gk"],
              gqd=w["gqd"], gkd=w["gkd"], seq_start=starts)
    native.mf_qk_rope_fwd(b["x"], b["y"], xd=b["xd"], yd=b["yd"], **rk)
    (q, k, v), (qd, kd, vd) = b["y"].split(COLS, 1), b["yd"].split(COLS, 1)
    (dq, dk, dv), (dqd, dkd, dvd) = b["dy"].split(COLS, 1), b["dyd"].split(COLS, 1)
    at = dict(n_heads=HQ, n_kv_heads=HKV, head_dim=D, window=WINDOW, n_sink=SINKS, qd=qd, kd=kd, vd=vd, od=b["od"],
              rbar=b["rbar"], seq_start=starts)
    native.mf_attn_window_fwd(q, k, v, b["o"], b["lse"], **at)
    native.mf_attn_window_bwd(q, k, v, b["o"], b["lse"], do, dq, dk, dv, work=b["work"][0], dod=dod, dqd=dqd, dkd=dkd,
                              dvd=dvd, **at)
    native.mf_qk_rope_bwd(b["dy"], b["dx"], x=b["x"], xd=b["xd"], dyd=b["dyd"], dxd=b["dxd"], work=b["work"][1],
                          dgq=b["dgq"], dgk=b["dgk"], dgqd=b["dgqd"], dgkd=b["dgkd"], **rk)
    native.mf_embed_bwd(ids, b["dx"], b["dE"], b["work"][2], scale=SCALE, dyd=b["dxd"], dEd=b["dEd"], seq_start=starts)


def _check(torch, w, ids, do, dod, lens, b):
    """Against the float64 composition.  Rows between the operators are bf16, so that each stage adds its
    roundings: a gradient passes through six (two of rows, P, dS, the attention's gradients, the result),
    2^-9 each in the mean square at most and amplified at most by the norms of what they multiply (about
    2): relative in the 2-norm 6 * 2^-9 * 2.  The embedding adds float32 roundings."""
    from oracle import packed as op
    n = sum(lens)
    pos, rates, pairs = op.positions(lens), op.rates(D), op.window_pairs(lens, WINDOW, SINKS)
    ids = ids[:n].long()
    pick = torch.zeros(n, V, dtype=torch.float64)
    real = ids >= 0
    pick[torch.arange(n)[real], ids[real]] = SCALE

    def f(E, gq, gk):
        r = op.qk_rope(pick @ E, gq, gk, HQ, HKV, D, pos, rates, "half")
        return op.masked_attention(*r.split(COLS, 1), HQ, HKV, D, pairs, D ** -0.5)[0]

    prim = tuple(w[k].double() for k in ("E", "gq", "gk"))
    tang = tuple(w[k].double() for k in ("Ed", "gqd", "gkd"))
    o, od = torch.func.jvp(f, prim, tang)
    gr, grd = op.grads_dual(f, prim, do[:n].double(), tang, dod[:n].double())
    for name, ref in (("o", o), ("od", od), ("dE", gr[0]), ("dEd", grd[0]), ("dgq", gr[1]), ("dgk", gr[2]),
                      ("dgqd", grd[1]), ("dgkd", grd[2])):
        got = b[name].double().cpu()
        got = got[:n] if name in ("o", "od") else got
        off = (got - ref).norm() / ref.norm()
        assert off <= 6 * 2.0 ** -9 * 2, (name, off.item())
    missing = torch.ones(V, dtype=torch.bool)
    missing[ids[real]] = False
    assert (b["dE"].cpu()[missing] == 0).all()


@pytest.mark.gpu
def test_embedding_to_windowed_attention_and_back():
    torch, native = need_gpu()
    lens = [190, 1, 77, 0, 620]
    N = sum(lens) + 9
    w = _weights(torch, 91)
    ids, do, dod = _tokens(torch, lens, N, 92)
    wc = {k: t.cuda() for k, t in w.items()}
    b = _buffers(torch, native, N)
    _run(native, wc, ids.cuda(), do.cuda(), dod.cuda(), au.starts_of(lens).cuda(), b)
    torch.cuda.synchronize()
    _check(torch, w, ids, do, dod, lens, b)


@pytest.mark.gpu
def test_captured_layer_with_other_tokens_and_lengths():
    torch, native = need_gpu()
    N = 700
    w = _weights(torch, 93)
    wc = {k: t.cuda() for k, t in w.items()}
    cur = [t.cuda() for t in _tokens(torch, [N], N, 94)]
    starts = torch.tensor([0, N, N, N], dtype=torch.int32, device="cuda")
    b = _buffers(torch, native, N)
    _run(native, wc, *cur, starts, b)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        _run(native, wc, *cur, starts, b)
    for seed, lens in ((95, [300, 20, 380]), (96, [13, 640]), (97, [0, 0, 90])):
        new = _tokens(torch, lens, N, seed)
        for a, t in zip(cur, new):
            a.copy_(t)
        s = au.starts_of(lens)
        starts.copy_(torch.cat([s, s[-1:].expand(4 - len(s))]))
        g.replay()
        torch.cuda.synchronize()
        _check(torch, w, *new, lens, b)
