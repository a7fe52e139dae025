"""Head norms with rotary positions (mf_qk_rope_fwd / mf_qk_rope_bwd) against the float64
definition: both layouts, partial rotation (also of parts that are no whole vector), scaled
rates, far positions, norms on and off, tangents, strided rows, the three type pairs, packed
sequences with rows behind the last one.

Tolerances.  The kernels work in float32 and round once, so an element is off by half a step
of its type relative to itself (bf16 2^-8) and by a small multiple of 2^-24 of the
magnitudes that it is summed from.  The longest chain is the tangent of the backward pass: five
products, two head sums of up to 128 terms added in a tree of eight-term chunks, angles good to
2^-22: 32 of 2^-24 covers each of its at most twelve terms, taken as 2^-17 of the row's largest
magnitude over all outputs of the head."""
import numpy as np
import pytest

from gpu_util import need_gpu
from oracle import packed as op

HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}
SUM = 2.0 ** -17

CASES = {
    # lens, tail, Hq, Hkv, copies, D, rope keywords, norm, x, y
    "one_token": ([1], 0, 1, 1, 0, 8, {}, True, "f32", "bf16"),
    "grouped": ([5, 0, 1, 40], 3, 4, 2, 2, 64, {}, True, "f32", "bf16"),
    "interleaved_part": ([17, 30], 0, 3, 1, 1, 128, dict(layout="interleaved", dims=64), True, "bf16", "bf16"),
    "half_part_odd": ([33], 2, 2, 2, 0, 24, dict(dims=10), True, "f32", "f32"),
    "interleaved_odd": ([9, 9], 0, 5, 1, 1, 40, dict(layout="interleaved", dims=14), True, "f32", "bf16"),
    "two_dims": ([12], 0, 2, 1, 1, 128, dict(dims=2), True, "f32", "f32"),
    "no_norm": ([64, 7], 0, 6, 3, 3, 80, dict(layout="interleaved"), False, "bf16", "bf16"),
    "no_norm_fp32": ([21], 1, 2, 2, 2, 96, dict(dims=48), False, "f32", "f32"),
    "linear": ([50], 0, 1, 1, 1, 64, dict(scaling="linear", factor=4.0), True, "f32", "f32"),
    "base": ([50], 0, 1, 1, 1, 64, dict(scaling="base", factor=8.0), True, "f32", "f32"),
    "bands": ([400], 0, 2, 1, 1, 64, dict(scaling="bands", factor=8.0, orig_len=128, low_turns=1.0,
                                         high_turns=4.0, mscale=1.25, base=500000.0), True, "f32", "f32"),
    "many_rows": ([3000, 1, 3501], 9, 4, 4, 4, 32, {}, True, "f32", "bf16"),
    "wide_rows": ([31], 0, 40, 8, 8, 128, {}, True, "bf16", "bf16"),
}
NAMES = [(n, d) for n in CASES for d in (False, True)]


def _data(name, dual, seed=0):
    lens, tail, Hq, Hkv, Hc, D, rk, norm, xt, yt = CASES[name]
    torch, native = need_gpu()
    dt = {"f32": torch.float32, "bf16": torch.bfloat16}
    g = torch.Generator().manual_seed(seed)
    N, W = sum(lens) + tail, (Hq + Hkv + Hc) * D

    def rnd(*s, std=1.0, t=torch.float32):
        return (torch.randn(*s, generator=g) * std).to(t)

    v = dict(x=rnd(N, W, t=dt[xt]), dy=rnd(N, W, t=dt[yt]))
    if dual:
        v.update(xd=rnd(N, W, std=0.5, t=dt[xt]), dyd=rnd(N, W, std=0.5, t=dt[yt]))
    if norm:
        v.update(gq=1 + rnd(D, std=0.2), gk=1 + rnd(D, std=0.2))
        if dual:
            v.update(gqd=rnd(D, std=0.3), gkd=rnd(D, std=0.3))
    starts = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
    return torch, native, v, torch.from_numpy(starts), dt[yt]


def _reference(name, dual, v, pos):
    import torch
    lens, tail, Hq, Hkv, Hc, D, rk, norm, xt, yt = CASES[name]
    n = len(pos)
    R = rk.get("dims") or D
    w = op.rates(R, rk.get("base", 10000.0), rk.get("scaling", "none"), rk.get("factor", 1.0),
                 rk.get("orig_len", 0), rk.get("low_turns", 1.0), rk.get("high_turns", 4.0))
    args = (Hq, Hkv, D, pos, w, rk.get("layout", "half"), rk.get("mscale", 1.0))
    z = {k: t.double() for k, t in v.items()}
    one = torch.ones(D, dtype=op.F64)
    if norm:
        f = lambda x, gq, gk: op.qk_rope(x, gq, gk, *args)
    else:
        f = lambda x, gq, gk: op.qk_rope(x, None, None, *args) + 0 * gq.sum() + 0 * gk.sum()
    prim = (z["x"][:n], z.get("gq", one), z.get("gk", one))
    out = {}
    if dual:
        tang = (z["xd"][:n], z.get("gqd", 0 * one), z.get("gkd", 0 * one))
        out["y"], out["yd"] = torch.func.jvp(f, prim, tang)
        g, gd = op.grads_dual(f, prim, z["dy"][:n], tang, z["dyd"][:n])
        out.update(dx=g[0], dgq=g[1], dgk=g[2], dxd=gd[0], dgqd=gd[1], dgkd=gd[2])
    else:
        out["y"] = f(*prim)
        g = op.grads(f, prim, z["dy"][:n])
        out.update(dx=g[0], dgq=g[1], dgk=g[2])
    return out


def _check(got, ref, half, what, D):
    """|got - ref| <= half |ref| + SUM max |ref| of the head (a row's whole head feeds each of
    its elements through the norm); at least of magnitude 1, which inputs and gains have."""
    import torch
    got, ref = got.double().cpu(), ref.cpu()
    top = ref.abs().unflatten(1, (-1, D)).amax(-1, keepdim=True).clamp_min(1.0).expand(-1, -1, D).flatten(1)
    off = (got - ref).abs() - (half * ref.abs() + SUM * top)
    assert torch.isfinite(got).all(), what
    assert off.max() <= 0, (what, off.max().item(), (got - ref).abs().max().item())


@pytest.mark.gpu
@pytest.mark.parametrize("name,dual", NAMES)
def test_rope_against_definition(name, dual):
    lens, tail, Hq, Hkv, Hc, D, rk, norm, xt, yt = CASES[name]
    torch, native, v, starts, ydt = _data(name, dual)
    pos = op.positions(lens)
    n, N = len(pos), len(pos) + tail
    ref = _reference(name, dual, v, pos)
    c = {k: t.cuda() for k, t in v.items()}
    W = (Hq + Hkv + Hc) * D
    kw = dict(n_heads=Hq, n_kv_heads=Hkv, head_dim=D, rope=native.rope_desc(**rk), n_copy_heads=Hc,
              gq=c.get("gq"), gk=c.get("gk"), gqd=c.get("gqd"), gkd=c.get("gkd"),
              seq_start=starts.cuda())
    # outputs are column ranges of wider rows, filled with a mark that has to survive behind
    # the last sequence and beside the columns
    mark = -7.0
    wide = {k: torch.full((N, W + 16), mark, dtype=ydt, device="cuda") for k in ("y", "yd", "dx", "dxd")}
    o = {k: t[:, 8:8 + W] for k, t in wide.items()}
    native.mf_qk_rope_fwd(c["x"], o["y"], xd=c.get("xd"), yd=o["yd"] if dual else None, **kw)
    dg = {k: torch.full((D,), mark, device="cuda") for k in ("dgq", "dgk", "dgqd", "dgkd")}
    work = torch.empty(native.mf_qk_rope_work_bytes(N, Hq, Hkv, D, dual), dtype=torch.uint8, device="cuda")
    use = {k: dg[k] for k in (("dgq", "dgk") if norm else ()) + (("dgqd", "dgkd") if norm and dual else ())}
    native.mf_qk_rope_bwd(c["dy"], o["dx"], x=c["x"] if norm else None,
                          xd=c.get("xd") if norm else None, dyd=c.get("dyd"),
                          dxd=o["dxd"] if dual else None, work=work, **use, **kw)
    torch.cuda.synchronize()
    for k in ("y", "dx") + (("yd", "dxd") if dual else ()):
        _check(o[k][:n], ref[k], HALF[yt], k, D)
        assert (wide[k][n:] == mark).all() and (wide[k][:, :8] == mark).all() \
            and (wide[k][:, 8 + W:] == mark).all(), k
    for k in use:
        # n * heads float32 terms of magnitude up to the largest: at most eight partial sums of
        # chains, each off by 2^-24 a step of what it holds; bounded by the sum of magnitudes
        terms = n * (Hq if k.startswith("dgq") else Hkv)
        bound = 2.0 ** -24 * 64 * (terms ** 0.5 + 8) * max(1.0, ref[k].abs().max().item())
        assert (dg[k].double().cpu() - ref[k]).abs().max() <= bound, k


@pytest.mark.gpu
@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_rope_far_and_negative_positions(layout):
    """Angles of positions up to 2^31 - 1 and below zero, as good as at position 0: the phase is
    exact modulo a turn up to the float64 rate's own 2^-53 (times 2^31 positions: 2^-22 turns,
    the only error that grows), and float32 cos and sin add 2^-22."""
    torch, native = need_gpu()
    pos = torch.tensor([0, 1, -1, 4095, 100000, 1234567, -1234567, 2 ** 31 - 1, -2 ** 31], dtype=torch.int32)
    D, n = 64, len(pos)
    x = torch.randn(n, 2 * D, generator=torch.Generator().manual_seed(1))
    y = torch.empty(n, 2 * D, device="cuda")
    native.mf_qk_rope_fwd(x.cuda(), y, 1, 1, D, native.rope_desc(layout=layout), pos=pos.cuda())
    ref = op.qk_rope(x.double(), None, None, 1, 1, D, pos, op.rates(D), layout)
    # the reference's own angles in float64: 2^31 * 2^-53 radians
    tol = (2.0 ** -21 + pos.double().abs()[:, None] * 2.0 ** -51) * 6.3 * x.abs().max()
    assert ((y.cpu().double() - ref).abs() <= tol).all(), (y.cpu().double() - ref).abs().max(1)


@pytest.mark.gpu
def test_rope_in_place_and_equal_sequences():
    """y = x, dx = dy, dx = x, and equal sequences given by their number."""
    torch, native = need_gpu()
    D, Hq, Hkv, B, S = 64, 4, 2, 3, 33
    g = torch.Generator().manual_seed(2)
    x = torch.randn(B * S, (Hq + 2 * Hkv) * D, generator=g).to(torch.bfloat16).cuda()
    gq = torch.rand(D, generator=g).cuda() + 0.5
    starts = torch.arange(B + 1, dtype=torch.int32).mul(S).cuda()
    r = native.rope_desc()
    kw = dict(n_heads=Hq, n_kv_heads=Hkv, head_dim=D, rope=r, n_copy_heads=Hkv, gq=gq, gk=gq)
    y = torch.empty_like(x)
    native.mf_qk_rope_fwd(x, y, seq_start=starts, **kw)
    z = x.clone()
    native.mf_qk_rope_fwd(z, z, n_seq=B, **kw)
    assert torch.equal(y, z)
    work = torch.empty(native.mf_qk_rope_work_bytes(B * S, Hq, Hkv, D), dtype=torch.uint8, device="cuda")
    out = []
    for dx, dy in ((torch.empty_like(y), y), (z, z), (x.clone(), y)):
        a, b = torch.empty(D, device="cuda"), torch.empty(D, device="cuda")
        native.mf_qk_rope_bwd(dy, dx, x=dx if torch.equal(dx, x) else x, dgq=a, dgk=b, work=work, n_seq=B, **kw)
        out.append((dx, a, b))
    for s, t, u in zip(*out):
        assert torch.equal(s, t) and torch.equal(s, u)


@pytest.mark.gpu
def test_rope_adjoint_identity():
    """<dy, y'> = <dx, x'> + <dg, g'>: the forward tangent and the backward pass are adjoint, in
    float32 (2^-24 a rounding, the sums of N W terms of random sign: 2^-16 of the norms)."""
    torch, native = need_gpu()
    N, Hq, Hkv, D = 257, 3, 2, 56
    g = torch.Generator().manual_seed(3)
    rnd = lambda *s: torch.randn(*s, generator=g).cuda()
    W = (Hq + Hkv) * D
    x, xd, dy = rnd(N, W), rnd(N, W), rnd(N, W)
    gs = dict(gq=rnd(D), gk=rnd(D))
    gt = dict(gqd=rnd(D), gkd=rnd(D))
    kw = dict(n_heads=Hq, n_kv_heads=Hkv, head_dim=D, rope=native.rope_desc(dims=40))
    y, yd, dx = (torch.empty(N, W, device="cuda") for _ in range(3))
    native.mf_qk_rope_fwd(x, y, xd=xd, yd=yd, **kw, **gs, **gt)
    dg = dict(dgq=torch.empty(D, device="cuda"), dgk=torch.empty(D, device="cuda"))
    work = torch.empty(native.mf_qk_rope_work_bytes(N, Hq, Hkv, D), dtype=torch.uint8, device="cuda")
    native.mf_qk_rope_bwd(dy, dx, x=x, work=work, **kw, **gs, **dg)
    dot = lambda a, b: (a.double() * b.double()).sum().item()
    left = dot(dy, yd)
    right = dot(dx, xd) + dot(dg["dgq"], gt["gqd"]) + dot(dg["dgk"], gt["gkd"])
    assert abs(left - right) <= 2.0 ** -16 * dy.double().norm().item() * yd.double().norm().item()


@pytest.mark.gpu
def test_rope_no_rows():
    torch, native = need_gpu()
    x = torch.zeros(0, 64, device="cuda")
    native.mf_qk_rope_fwd(x, x, 1, 1, 32, native.rope_desc())
    d = [torch.full((32,), 3.0, device="cuda") for _ in range(2)]
    work = torch.empty(native.mf_qk_rope_work_bytes(0, 1, 1, 32), dtype=torch.uint8, device="cuda")
    one = torch.ones(32, device="cuda")
    native.mf_qk_rope_bwd(x, x, 1, 1, 32, native.rope_desc(), x=x, gq=one, gk=one, dgq=d[0],
                          dgk=d[1], work=work)
    # rows, but none of them in a sequence
    y = torch.full((5, 64), 2.0, device="cuda")
    dz = [torch.full((32,), 3.0, device="cuda") for _ in range(2)]
    native.mf_qk_rope_bwd(y, y, 1, 1, 32, native.rope_desc(), x=y, gq=one, gk=one, dgq=dz[0],
                          dgk=dz[1], work=work, seq_start=torch.zeros(2, dtype=torch.int32, device="cuda"))
    for t in d + dz:
        assert (t == 0).all()
    assert (y == 2.0).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dual", [False, True])
def test_rope_not_finite_stays_in_its_head(dual):
    """A NaN or an infinity in one head reaches that head's own outputs and gains alone: not the
    other kind of heads' gains, nor any other head or row."""
    torch, native = need_gpu()
    N, Hq, Hkv, D = 9, 3, 2, 40
    g = torch.Generator().manual_seed(4)
    rnd = lambda *s: torch.randn(*s, generator=g).cuda()
    W = (Hq + 2 * Hkv) * D
    base = {k: rnd(N, W) for k in ("x", "dy") + (("xd", "dyd") if dual else ())}
    gains = dict(gq=rnd(D), gk=rnd(D), **(dict(gqd=rnd(D), gkd=rnd(D)) if dual else {}))
    names = ["dgq", "dgk"] + ["dgqd", "dgkd"] * dual
    work = torch.empty(native.mf_qk_rope_work_bytes(N, Hq, Hkv, D, dual), dtype=torch.uint8, device="cuda")

    def run(v):
        kw = dict(n_heads=Hq, n_kv_heads=Hkv, head_dim=D, rope=native.rope_desc(), n_copy_heads=Hkv, **gains)
        o = {k: torch.empty(N, W, device="cuda") for k in ("y", "dx") + (("yd", "dxd") if dual else ())}
        dg = {k: torch.empty(D, device="cuda") for k in names}
        native.mf_qk_rope_fwd(v["x"], o["y"], xd=v.get("xd"), yd=o.get("yd"), **kw)
        native.mf_qk_rope_bwd(v["dy"], o["dx"], x=v["x"], xd=v.get("xd"), dyd=v.get("dyd"),
                              dxd=o.get("dxd"), work=work, **dg, **kw)
        return o, dg

    ref, dref = run(base)
    for head, val in ((1, float("nan")), (Hq, float("inf")), (Hq + Hkv, float("nan"))):
        for name in base:
            v = {k: t.clone() for k, t in base.items()}
            v[name][4, head * D + 7] = val
            o, dg = run(v)
            for k in o:
                other = torch.ones(N, W, dtype=torch.bool, device="cuda")
                other[4, head * D:(head + 1) * D] = False
                assert torch.equal(o[k][other], ref[k][other]), (head, name, k)
            for k in names:
                kind = 0 if k.startswith("dgq") else 1
                mine = 0 if head < Hq else 1 if head < Hq + Hkv else 2
                if kind != mine:
                    assert torch.equal(dg[k], dref[k]), (head, name, k)


@pytest.mark.gpu
def test_rope_captured_with_other_lengths():
    """Both passes in one graph, replayed after the starts have changed on the device."""
    torch, native = need_gpu()
    N, Hq, Hkv, D = 300, 4, 2, 64
    g = torch.Generator().manual_seed(8)
    x, dy = (torch.randn(N, (Hq + 2 * Hkv) * D, generator=g).cuda() for _ in range(2))
    gains = dict(gq=torch.rand(D, generator=g).cuda() + 0.5, gk=torch.rand(D, generator=g).cuda() + 0.5)
    starts = torch.tensor([0, 100, 300], dtype=torch.int32, device="cuda")
    work = torch.empty(native.mf_qk_rope_work_bytes(N, Hq, Hkv, D), dtype=torch.uint8, device="cuda")

    def run(o):
        kw = dict(n_heads=Hq, n_kv_heads=Hkv, head_dim=D, rope=native.rope_desc(), n_copy_heads=Hkv,
                  seq_start=starts, **gains)
        native.mf_qk_rope_fwd(x, o["y"], **kw)
        native.mf_qk_rope_bwd(dy, o["dx"], x=x, dgq=o["dgq"], dgk=o["dgk"], work=work, **kw)

    def outs():
        o = {k: torch.zeros_like(x) for k in ("y", "dx")}
        return {**o, **{k: torch.zeros(D, device="cuda") for k in ("dgq", "dgk")}}

    run(outs())
    torch.cuda.synchronize()
    o, graph = outs(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run(o)
    for s in ([0, 100, 300], [0, 7, 260], [0, 0, 1]):
        starts.copy_(torch.tensor(s, dtype=torch.int32))
        for t in o.values():
            t.zero_()
        graph.replay()
        want = outs()
        run(want)
        torch.cuda.synchronize()
        for k in o:
            assert torch.equal(o[k], want[k]), (s, k)
