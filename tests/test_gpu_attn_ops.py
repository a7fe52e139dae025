"""Packed causal attention with grouped heads (mf_attn_fwd / mf_attn_bwd) against the float64
definition, element by element within bounds derived from the roundings (attn_ops_util):
sequence lengths of zero, one and around every tile edge, head widths that fill no tile,
grouped heads, tangents, strided rows, rows behind the last sequence, non-finite values in
masked places, streams, graphs."""
import math

import pytest

import attn_ops_util as au
from gpu_util import need_gpu

CASES = {
    # lens, tail, Hq, Hkv, D
    "one_token": ([1], 0, 1, 1, 64),
    "one_and_32": ([1, 32], 0, 4, 2, 32),
    "narrow": ([9, 30], 1, 2, 1, 8),
    "tile": ([128], 0, 2, 2, 64),
    "past_tile": ([129], 3, 2, 1, 64),
    "edges": ([64, 0, 65, 1, 127, 128, 3], 5, 4, 2, 64),
    "ragged": ([300, 1, 1, 211, 0, 63], 130, 4, 1, 64),
    "odd_width": ([200, 77], 0, 3, 3, 40),
    "many_short": ([3, 5, 1, 7, 2, 9, 4, 4, 8, 6, 1, 1, 30, 17, 2, 90, 12], 2, 2, 2, 16),
    "long": ([700], 0, 2, 1, 64),
    # groups that one cluster shares whole: eight, six, seven and ten heads
    "group_8": ([260, 40], 0, 8, 1, 32),
    "group_6": ([131, 5], 3, 6, 1, 64),
    "group_7_of_2": ([90, 60], 0, 14, 2, 64),
    "group_10": ([140], 0, 10, 1, 24),
    # so many CTAs that tiles of 64 keys are taken
    "many_heads": ([300, 1, 128, 211, 0, 400, 353, 400], 2, 64, 8, 64),
    # more sequences than a block reads at once
    "many_sequences": ([0, 1, 2, 0, 1, 3] * 380, 1, 2, 1, 16),
}
WIDE = {
    "wide_one": ([1], 0, 2, 1, 128),
    "wide_72": ([130, 66], 1, 2, 2, 72),
    "wide_edges": ([128, 1, 0, 255, 64], 7, 4, 2, 128),
    "wide_long": ([600, 40], 0, 3, 1, 128),
    "wide_96_grouped": ([190], 0, 8, 1, 96),
}
RUNS = [(n, d) for n in CASES for d in (False, True)] + [(n, False) for n in WIDE]


@pytest.mark.gpu
@pytest.mark.parametrize("name,dual", RUNS)
def test_attention_against_definition(name, dual):
    torch, native = need_gpu()
    lens, tail, Hq, Hkv, D = {**CASES, **WIDE}[name]
    v = au.data(lens, tail, Hq, Hkv, D, dual)
    ref, bound = au.reference(v, lens, Hq, Hkv, D)
    out = au.run(native, au.wide(v), lens, Hq, Hkv, D)
    torch.cuda.synchronize()
    au.check(out, ref, bound, sum(lens), dual)


@pytest.mark.gpu
@pytest.mark.parametrize("D,dual", [(64, False), (64, True), (128, False)])
def test_attention_large_scores_and_scale(D, dual):
    """Scores of several hundred: softmax rows that are one key, statistics far from zero."""
    torch, native = need_gpu()
    lens, Hq, Hkv = [150, 90], 2, 1
    v = au.data(lens, 0, Hq, Hkv, D, dual, seed=5, qstd=12.0)
    ref, bound = au.reference(v, lens, Hq, Hkv, D, scale=0.75)
    out = au.run(native, au.wide(v), lens, Hq, Hkv, D, scale=0.75)
    torch.cuda.synchronize()
    assert ref["lse"].abs().max() > 300
    au.check(out, ref, bound, sum(lens), dual)


@pytest.mark.gpu
@pytest.mark.parametrize("D,dual", [(64, False), (64, True), (128, False), (40, True)])
@pytest.mark.parametrize("poison", [math.nan, math.inf, -math.inf])
def test_attention_masked_places_do_not_matter(D, dual, poison):
    """Values of rows that a row does not attend to never reach it: those behind the last
    sequence, those of other sequences, and later ones of its own."""
    torch, native = need_gpu()
    lens, tail, Hq, Hkv = [70, 45, 100, 20], 33, 2, 1
    n = sum(lens)
    clean = au.data(lens, tail, Hq, Hkv, D, dual, seed=6)
    want = {k: t.clone() for k, t in au.run(native, au.wide(clean), lens, Hq, Hkv, D).items()}
    # rows behind the last sequence, the whole second sequence, and the last row of the third
    bad = list(range(70, 115)) + [214] + list(range(n, n + tail))
    dirty = {k: t.clone() for k, t in clean.items()}
    for t in dirty.values():
        t[bad] = poison
    got = au.run(native, au.wide(dirty), lens, Hq, Hkv, D)
    torch.cuda.synchronize()
    assert int(got["status"].item()) == 0
    ahead = torch.tensor([r for r in range(n) if r not in bad])
    # forward: every other row, bit for bit
    for k in au.names(dual, False):
        a, b = (got[k].t(), want[k].t()) if k in ("lse", "rbar") else (got[k], want[k])
        assert torch.equal(a[ahead.cuda()], b[ahead.cuda()]), k
        assert not torch.isfinite(a[70:115]).all(1).any(), k     # a poisoned row shows it
    # backward: dq of every other row; dk, dv where no poisoned row attends (the third
    # sequence's rows are attended to by its poisoned last row)
    clear = torch.tensor(list(range(70)) + list(range(215, n))).cuda()
    for k in au.names(dual)[len(au.names(dual, False)):]:
        rows = ahead.cuda() if k.startswith("dq") else clear
        assert torch.equal(got[k][rows], want[k][rows]), k
        assert (got[k][n:] == au.MARK).all(), k
        if not k.startswith("dq"):
            assert not torch.isfinite(got[k][115:215]).all(1).any(), k


@pytest.mark.gpu
def test_attention_masked_places_do_not_matter_many_heads():
    """The same where there are so many CTAs that tiles of 64 keys are taken."""
    torch, native = need_gpu()
    lens, tail, Hq, Hkv, D = [70, 45, 100, 20], 33, 320, 1, 24
    n = sum(lens)
    clean = au.data(lens, tail, Hq, Hkv, D, False, seed=6)
    want = {k: t.clone() for k, t in au.run(native, au.wide(clean), lens, Hq, Hkv, D).items()}
    dirty = {k: t.clone() for k, t in clean.items()}
    bad = list(range(70, 115)) + list(range(n, n + tail))
    for t in dirty.values():
        t[bad] = math.nan
    got = au.run(native, au.wide(dirty), lens, Hq, Hkv, D)
    torch.cuda.synchronize()
    rest = torch.tensor([r for r in range(n) if r not in bad]).cuda()
    for k in ("o", "dq", "dk", "dv"):
        assert torch.equal(got[k][rest], want[k][rest]), k
    assert torch.equal(got["lse"][:, rest], want["lse"][:, rest])


@pytest.mark.gpu
@pytest.mark.parametrize("D,dual", [(64, True), (128, False)])
def test_attention_two_calls_at_once(D, dual):
    """Calls that overlap on two streams, each with its own workspace, do not meet."""
    torch, native = need_gpu()
    jobs = []
    for seed, lens in ((1, [700, 90]), (2, [64, 400, 333])):
        v = au.wide(au.data(lens, 0, 4, 2, D, dual, seed=seed))
        jobs.append((v, lens, {k: t.clone() for k, t in au.run(native, v, lens, 4, 2, D).items()}))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in jobs]
    for _ in range(20):
        outs = []
        for (v, lens, _), s in zip(jobs, streams):
            with torch.cuda.stream(s):
                outs.append(au.run(native, v, lens, 4, 2, D))
        torch.cuda.synchronize()
        for (v, lens, want), got in zip(jobs, outs):
            for k in au.names(dual):
                assert torch.equal(got[k], want[k]), k


@pytest.mark.gpu
@pytest.mark.parametrize("dual", [False, True])
def test_rows_far_apart(dual):
    """Elements behind the 2^31st of a buffer: the same bits as from rows close together."""
    torch, native = need_gpu()
    N, Hq, Hkv, D = 9000, 2, 1, 32
    lens = [4000, 1, 4999]
    W = (Hq + 2 * Hkv) * D
    far = torch.empty(N, 245760, dtype=torch.bfloat16, device="cuda")      # 2.2e9 elements
    v = {k: t.cuda() for k, t in au.data(lens, 0, Hq, Hkv, D, dual).items()}
    want = au.run(native, v, lens, Hq, Hkv, D)
    at = 245760 - 8
    def put(cols):
        nonlocal at
        at -= cols
        return far[:, at:at + cols]
    apart = {}
    for k, t in v.items():
        apart[k] = put(t.shape[1])
        apart[k].copy_(t)
    out = {k: (put(t.shape[1]) if t.dtype is torch.bfloat16 and t.shape[0] == N else t.clone())
           for k, t in want.items()}
    got = au.run(native, apart, lens, Hq, Hkv, D, out=out)
    for k in au.names(dual):
        assert torch.equal(got[k], want[k]), k
    # the head norms between rows as far apart
    x = torch.cat([v["q"], v["k"], v["v"]], 1)
    kw = dict(n_heads=Hq, n_kv_heads=Hkv, head_dim=D, rope=native.rope_desc(), n_copy_heads=Hkv,
              gq=torch.ones(D, device="cuda"), gk=torch.ones(D, device="cuda"),
              seq_start=au.starts_of(lens).cuda())
    y = torch.empty_like(x)
    native.mf_qk_rope_fwd(x, y, **kw)
    xf, yf = put(W), put(W)
    xf.copy_(x)
    native.mf_qk_rope_fwd(xf, yf, **kw)
    assert torch.equal(yf, y)


@pytest.mark.gpu
@pytest.mark.parametrize("D,dual", [(64, True), (128, False)])
def test_attention_same_bits_again_and_on_another_stream(D, dual):
    torch, native = need_gpu()
    lens, tail, Hq, Hkv = [333, 64, 190], 4, 4, 2
    v = au.wide(au.data(lens, tail, Hq, Hkv, D, dual, seed=7))
    first = {k: t.clone() for k, t in au.run(native, v, lens, Hq, Hkv, D).items()}
    again = au.run(native, v, lens, Hq, Hkv, D)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    third = au.run(native, v, lens, Hq, Hkv, D, starts=au.starts_of(lens).cuda(), stream=side)
    torch.cuda.synchronize()
    for k in au.names(dual):
        assert torch.equal(first[k], again[k]) and torch.equal(first[k], third[k]), k


@pytest.mark.gpu
@pytest.mark.parametrize("D,dual", [(64, True), (128, False)])
def test_attention_captured_with_other_lengths(D, dual):
    """A captured call replayed after the lengths on the device have changed (fewer rows too)."""
    torch, native = need_gpu()
    Hq, Hkv, N = 2, 1, 300
    sets = [[300], [10, 200, 90], [150, 0, 50]]
    v = au.data([N], 0, Hq, Hkv, D, dual, seed=8)
    w = au.wide(v)
    starts = torch.zeros(4, dtype=torch.int32, device="cuda")

    def put(lens):
        s = au.starts_of(lens)
        full = torch.cat([s, s[-1:].expand(4 - len(s))])
        starts.copy_(full)

    put(sets[0])
    out = au.run(native, w, None, Hq, Hkv, D, starts=starts)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        au.run(native, w, None, Hq, Hkv, D, starts=starts, out=out)
    for lens in sets:
        put(lens)
        for k in au.names(dual):
            out[k].fill_(au.MARK)
        g.replay()
        torch.cuda.synchronize()
        n = sum(lens)
        ref, bound = au.reference({k: t[:n] for k, t in v.items()}, lens, Hq, Hkv, D)
        au.check(out, ref, bound, n, dual)


@pytest.mark.gpu
@pytest.mark.parametrize("D", [64, 48])
def test_attention_adjoint_identity(D):
    """<do, o'> = <dq, q'> + <dk, k'> + <dv, v'>: the forward tangent against the backward
    pass.  Both sides carry roundings of 2^-8 with random signs over N Hq D terms; the sum of
    that many is within 2^-8 of the product of the norms."""
    torch, native = need_gpu()
    lens, Hq, Hkv = [211, 130], 4, 2
    v = au.wide(au.data(lens, 0, Hq, Hkv, D, True, seed=9))
    o = au.run(native, v, lens, Hq, Hkv, D)
    dot = lambda a, b: (a.double() * b.double()).sum().item()
    left = dot(v["do"], o["od"])
    right = dot(o["dq"], v["qd"]) + dot(o["dk"], v["kd"]) + dot(o["dv"], v["vd"])
    size = v["do"].double().norm().item() * o["od"].double().norm().item()
    assert abs(left - right) <= 2.0 ** -8 * size, (left, right, size)


@pytest.mark.gpu
def test_attention_sequences_out_of_order_stay_inside():
    """seq_start is read on the device and cannot be refused: wrong contents give undefined
    rows, but no access outside the buffers and no endless walk (every index is clamped)."""
    torch, native = need_gpu()
    Hq, Hkv, D, N = 2, 1, 64, 260
    v = au.wide(au.data([N], 0, Hq, Hkv, D, True, seed=10))
    for s in ([0, 200, 100, 260], [5, -7, 10 ** 9, 2 ** 31 - 1], [0, 0, 0, -5], [300, 300, 300, 260]):
        starts = torch.tensor(s, dtype=torch.int32, device="cuda")
        out = au.run(native, v, None, Hq, Hkv, D, starts=starts)
        torch.cuda.synchronize()
        assert int(out["status"].item()) == 0


@pytest.mark.gpu
def test_attention_no_rows():
    torch, native = need_gpu()
    for N in (0, 40):
        v = au.wide(au.data([0], N, 2, 1, 64, True, seed=11))
        out = au.run(native, v, [0], 2, 1, 64)
        torch.cuda.synchronize()
        au.check(out, {}, {}, 0, True)


@pytest.mark.gpu
def test_rope_then_attention_as_a_layer():
    """The operators as a transformer block calls them: projection rows (float32) through norm
    and rotary positions into the attention, its gradients back through them, with tangents,
    against the float64 composition.  Intermediate rows are bf16, so each stage adds its
    roundings: the gradient passes through six (two of rows, P, dS, the attention's gradients,
    the result), 2^-8 each at most and amplified at most by the norms of what they multiply
    (about 2 for unit-variance operands): within 2^-8 * 12 of the largest entry, relative in the
    2-norm 6 * 2^-9 * 2."""
    from oracle import packed as op
    torch, native = need_gpu()
    lens, Hq, Hkv, D = [190, 1, 77], 4, 2, 64
    N, W = sum(lens), (Hq + 2 * Hkv) * D
    g = torch.Generator().manual_seed(12)
    rnd = lambda *s, std=1.0: torch.randn(*s, generator=g) * std
    x, xd = rnd(N, W), rnd(N, W, std=0.5)
    gs = [1 + rnd(D, std=0.2) for _ in range(2)]
    gt = [rnd(D, std=0.2) for _ in range(2)]
    do, dod = rnd(N, Hq * D).bfloat16(), rnd(N, Hq * D, std=0.5).bfloat16()
    pos, w = op.positions(lens), op.rates(D)
    c = lambda t: t.cuda()
    starts = au.starts_of(lens).cuda()
    rk = dict(n_heads=Hq, n_kv_heads=Hkv, head_dim=D, rope=native.rope_desc(), n_copy_heads=Hkv,
              gq=c(gs[0]), gk=c(gs[1]), gqd=c(gt[0]), gkd=c(gt[1]), seq_start=starts)
    y, yd = (torch.empty(N, W, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    xc, xdc = c(x), c(xd)
    native.mf_qk_rope_fwd(xc, y, xd=xdc, yd=yd, **rk)
    cols = [Hq * D, Hkv * D, Hkv * D]
    v = dict(zip(("q", "k", "v"), y.split(cols, 1)))
    v.update(zip(("qd", "kd", "vd"), yd.split(cols, 1)))
    v.update(do=c(do), dod=c(dod))
    dy, dyd = torch.empty_like(y), torch.empty_like(y)
    out = dict(zip(("dq", "dk", "dv"), dy.split(cols, 1)))
    out.update(zip(("dqd", "dkd", "dvd"), dyd.split(cols, 1)))
    for k in ("o", "od"):
        out[k] = torch.empty(N, Hq * D, dtype=torch.bfloat16, device="cuda")
    for k in ("lse", "rbar"):
        out[k] = torch.empty(Hq, N, device="cuda")
    out["work"] = torch.empty(native.mf_attn_work_bytes(N, Hq, True), dtype=torch.uint8, device="cuda")
    out["status"] = torch.zeros(1, dtype=torch.int32, device="cuda")
    au.run(native, v, lens, Hq, Hkv, D, starts=starts, out=out)
    dx, dxd = torch.empty_like(y), torch.empty_like(y)
    dg = {k: torch.empty(D, device="cuda") for k in ("dgq", "dgk", "dgqd", "dgkd")}
    work = torch.empty(native.mf_qk_rope_work_bytes(N, Hq, Hkv, D, True), dtype=torch.uint8, device="cuda")
    native.mf_qk_rope_bwd(dy, dx, x=xc, xd=xdc, dyd=dyd, dxd=dxd, work=work, **dg, **rk)
    torch.cuda.synchronize()

    def f(x, gq, gk):
        r = op.qk_rope(x, gq, gk, Hq, Hkv, D, pos, w, "half")
        return op.attention(*r.split(cols, 1), Hq, Hkv, D, lens, D ** -0.5)[0]

    prim = (x.double(), gs[0].double(), gs[1].double())
    tang = (xd.double(), gt[0].double(), gt[1].double())
    o, od = torch.func.jvp(f, prim, tang)
    gr, grd = op.grads_dual(f, prim, do.double(), tang, dod.double())
    tol = 6 * 2.0 ** -9 * 2
    for got, ref in ((out["o"], o), (out["od"], od), (dx, gr[0]), (dxd, grd[0]), (dg["dgq"], gr[1]),
                     (dg["dgk"], gr[2]), (dg["dgqd"], grd[1]), (dg["dgkd"], grd[2])):
        off = (got.double().cpu() - ref).norm() / ref.norm()
        assert off <= tol, off
