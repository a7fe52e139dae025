"""Operators on packed token rows without a GPU: refusals of the C entry points and of the
binding, and the float64 definitions that the GPU tests compare with, checked against
differences."""
import ctypes as C
import math

import pytest
import torch

import attn_ops_util as au
from oracle import packed as op


@pytest.fixture(scope="module")
def native():
    from paper_2505_00793_gb300 import build, native
    build.build()
    return native


OK, INVALID, UNSUPPORTED = 0, 1, 2
P = 4096   # a pointer that no refused call reads


def _rope(native, **kw):
    a = native.mf_qk_rope_args()
    a.n_rows, a.n_heads, a.n_kv_heads, a.n_copy_heads, a.head_dim = 8, 2, 1, 1, 64
    a.x_prec = a.y_prec = 1
    a.eps, a.n_seq = 1e-6, 1
    a.rope = native.rope_desc()
    for i, k in enumerate(("x", "y", "dy", "dx", "gq", "gk", "dgq", "dgk", "work")):
        setattr(a, k, P * (1 + i))
    a.ldx = a.ldy = a.lddy = a.lddx = 256
    a.work_bytes = 1 << 30
    for k, v in kw.items():
        setattr(a, k, v)
    return a


ROPE_BAD = [
    dict(n_rows=-1), dict(n_rows=2 ** 31), dict(n_heads=0), dict(n_kv_heads=0), dict(n_copy_heads=-1),
    dict(head_dim=0), dict(head_dim=4), dict(head_dim=12), dict(head_dim=136), dict(x_prec=2),
    dict(y_prec=-1), dict(eps=-1.0), dict(eps=math.nan), dict(ldx=184), dict(ldx=257), dict(x=None),
    dict(x=P + 8), dict(gq=None), dict(gk=None), dict(gqd=P), dict(gkd=P), dict(gqd=P, gkd=P),
    dict(n_seq=0), dict(n_seq=-1), dict(n_seq=3), dict(gq=P + 4), dict(ldx=1 << 40),
]
DESC_BAD = [
    dict(layout=2), dict(layout=-1), dict(dims=3), dict(dims=66), dict(dims=-2), dict(base=-1.0),
    dict(base=math.inf), dict(mscale=math.nan), dict(scaling=4), dict(scaling=1, factor=0.0),
    dict(scaling=2, factor=-2.0), dict(scaling=2, factor=2.0, dims=2),
    dict(scaling=3, factor=2.0, orig_len=0, low_turns=1.0, high_turns=4.0),
    dict(scaling=3, factor=2.0, orig_len=8, low_turns=4.0, high_turns=4.0),
    dict(scaling=3, factor=2.0, orig_len=8, low_turns=-1.0, high_turns=4.0),
    dict(scaling=3, factor=2.0, orig_len=8, low_turns=math.nan, high_turns=4.0),
]


@pytest.mark.parametrize("kw", ROPE_BAD, ids=str)
def test_rope_refuses(native, kw):
    for f in ("mf_qk_rope_fwd", "mf_qk_rope_bwd"):
        assert getattr(native.lib(), f)(C.byref(_rope(native, **kw)), None) == INVALID, f


@pytest.mark.parametrize("kw", DESC_BAD, ids=str)
def test_rope_refuses_descriptor(native, kw):
    a = _rope(native)
    for k, v in kw.items():
        setattr(a.rope, k, v)
    for f in ("mf_qk_rope_fwd", "mf_qk_rope_bwd"):
        assert getattr(native.lib(), f)(C.byref(a), None) == INVALID, f


def test_rope_refuses_per_pass(native):
    L = native.lib()
    fwd = [dict(y=None), dict(y=P + 2), dict(ldy=8), dict(xd=P), dict(yd=P), dict(xd=P, yd=2 * P + 8),
           dict(y=P, ldy=264)]
    bwd = [dict(dy=None), dict(dx=None), dict(lddx=8), dict(dyd=P), dict(dxd=P), dict(dgq=None),
           dict(work=None), dict(work=P + 8), dict(work_bytes=64), dict(dyd=P, dxd=2 * P),
           dict(dyd=P, dxd=2 * P, xd=P, dgqd=P), dict(dx=P, lddx=264)]
    for kw in fwd:
        assert L.mf_qk_rope_fwd(C.byref(_rope(native, **kw)), None) == INVALID, kw
    for kw in bwd:
        assert L.mf_qk_rope_bwd(C.byref(_rope(native, **kw)), None) == INVALID, kw
    a = _rope(native, x_prec=1, y_prec=0)
    assert L.mf_qk_rope_fwd(C.byref(a), None) == UNSUPPORTED
    assert L.mf_qk_rope_fwd(C.byref(_rope(native, x_prec=0, y_prec=1, y=P)), None) == INVALID   # in place
    for f in (L.mf_qk_rope_fwd, L.mf_qk_rope_bwd, L.mf_attn_fwd, L.mf_attn_bwd):
        assert f(None, None) == INVALID
    assert L.mf_qk_rope_fwd(C.byref(_rope(native, n_rows=0, x=None)), None) == OK


def _attn(native, **kw):
    a = native.mf_attn_args()
    a.n_rows, a.n_heads, a.n_kv_heads, a.head_dim, a.n_seq = 8, 4, 2, 64, 1
    for i, k in enumerate(("q", "k", "v", "o", "lse", "d_o", "dq", "dk", "dv", "work")):
        setattr(a, k, P * (1 + i))
    for k in ("ldq", "ldk", "ldv", "ldo", "lddo", "lddq", "lddk", "lddv"):
        setattr(a, k, 256)
    a.work_bytes = 1 << 30
    for k, v in kw.items():
        setattr(a, k, v)
    return a


DUAL = {k: P * (20 + i) for i, k in enumerate(("qd", "kd", "vd", "od", "rbar", "d_od", "dqd", "dkd", "dvd"))}
ATTN_BAD = [
    dict(n_rows=-1), dict(n_rows=2 ** 31), dict(n_heads=0), dict(n_heads=3), dict(n_kv_heads=0),
    dict(head_dim=0), dict(head_dim=60), dict(head_dim=136), dict(scale=-1.0), dict(scale=math.inf),
    dict(scale=math.nan), dict(n_seq=0), dict(n_seq=3), dict(q=None), dict(k=None), dict(v=None),
    dict(o=None), dict(lse=None), dict(q=P + 8), dict(ldq=248), dict(ldk=120), dict(ldv=260),
    dict(ldo=0), dict(ldq=-256), dict(ldk=1 << 40),
] + [dict({k: None}, **{j: DUAL[j] for j in DUAL if j != k}) for k in ("qd", "kd", "vd", "od", "rbar")] \
  + [dict(DUAL, kd=P + 2)]
ATTN_BWD_BAD = [dict(d_o=None), dict(dq=None), dict(dk=P + 4), dict(dv=None), dict(work=None),
                dict(work=P + 8), dict(work_bytes=127), dict(lddo=8), dict(lddq=248), dict(lddk=4),
                dict(lddv=130), dict(DUAL, d_od=None), dict(DUAL, dqd=None), dict(DUAL, work_bytes=255),
                dict(dkd=DUAL["dkd"])]


@pytest.mark.parametrize("kw", ATTN_BAD, ids=str)
def test_attention_refuses(native, kw):
    for f in ("mf_attn_fwd", "mf_attn_bwd"):
        assert getattr(native.lib(), f)(C.byref(_attn(native, **kw)), None) == INVALID, f


@pytest.mark.parametrize("kw", ATTN_BWD_BAD, ids=str)
def test_attention_backward_refuses(native, kw):
    assert native.lib().mf_attn_bwd(C.byref(_attn(native, **kw)), None) == INVALID


@pytest.mark.parametrize("out,other", [("o", "q"), ("o", "v"), ("od", "o"), ("od", "kd"), ("o", "lse")])
def test_attention_refuses_outputs_over_others(native, out, other):
    kw = dict(DUAL)
    base = _attn(native, **kw)
    a = _attn(native, **{**kw, out: getattr(base, other)})
    assert native.lib().mf_attn_fwd(C.byref(a), None) == INVALID


@pytest.mark.parametrize("out,other", [("dq", "q"), ("dk", "dv"), ("dv", "d_o"), ("dqd", "dq"), ("dkd", "k"),
                                       ("work", "o"), ("dq", "o"), ("dvd", "od")])
def test_attention_backward_refuses_outputs_over_others(native, out, other):
    base = _attn(native, **DUAL)
    a = _attn(native, **{**DUAL, out: getattr(base, other)})
    assert native.lib().mf_attn_bwd(C.byref(a), None) == INVALID


def test_rope_refuses_outputs_over_others(native):
    """In place is y = x, yd = xd, dx = dy or x, dxd = dyd or xd; nothing else."""
    L, t = native.lib(), dict(xd=P * 30, yd=P * 31, dyd=P * 32, dxd=P * 33, dgqd=P * 34, dgkd=P * 35)
    base = _rope(native, **t)
    for out, other in (("yd", "y"), ("y", "xd"), ("yd", "x")):
        assert L.mf_qk_rope_fwd(C.byref(_rope(native, **{**t, out: getattr(base, other)})), None) == INVALID
    for out, other in (("dxd", "dx"), ("dx", "xd"), ("dxd", "dy"), ("dgq", "dgk"), ("dgqd", "gq"), ("work", "dx")):
        assert L.mf_qk_rope_bwd(C.byref(_rope(native, **{**t, out: getattr(base, other)})), None) == INVALID
    assert L.mf_qk_rope_bwd(C.byref(_rope(native, dx=base.x, lddx=264)), None) == INVALID
    assert L.mf_qk_rope_bwd(C.byref(_rope(native, dx=base.x, x_prec=0)), None) == INVALID


def test_attention_refuses_wide_tangents(native):
    a = _attn(native, head_dim=72, ldq=512, ldk=512, ldv=512, ldo=512, **DUAL)
    assert native.lib().mf_attn_fwd(C.byref(a), None) == UNSUPPORTED


def test_work_bytes(native):
    assert native.mf_attn_work_bytes(10, 3) == 120
    assert native.mf_attn_work_bytes(10, 3, True) == 240
    assert native.mf_qk_rope_work_bytes(10, 2, 1, 64, True) == 2 * native.mf_qk_rope_work_bytes(10, 2, 1, 64)
    with pytest.raises(native.MixflowError):
        native.mf_attn_work_bytes(-1, 3)


def test_binding_refuses(native):
    with pytest.raises(ValueError, match="layout"):
        native.rope_desc(layout="other")
    with pytest.raises(ValueError, match="scaling"):
        native.rope_desc(scaling="other")
    x = torch.zeros(4, 192)
    with pytest.raises(ValueError, match="CUDA"):
        native.mf_qk_rope_fwd(x, x, 1, 1, 64, native.rope_desc())
    b = x.bfloat16()
    with pytest.raises(ValueError, match="CUDA"):
        native.mf_attn_fwd(b, b, b, b, torch.zeros(1, 4), 1, 1, 64)


def _central(f, prim, tang, e=1e-5):
    up = f(*[p + e * t for p, t in zip(prim, tang)])
    dn = f(*[p - e * t for p, t in zip(prim, tang)])
    return (up - dn) / (2 * e)


def test_definitions_against_differences():
    """Tangents of the float64 definitions, and tangents of their gradients, against central
    differences (error e^2 of the third derivative plus 2^-52 / e of the values)."""
    g = torch.Generator().manual_seed(0)
    rnd = lambda *s: torch.randn(*s, generator=g, dtype=torch.float64)
    lens, Hq, Hkv, D = [5, 1, 4], 2, 1, 6
    N = sum(lens)
    rope = lambda x, a, b: op.qk_rope(x, a, b, Hq, Hkv, D, op.positions(lens), op.rates(4), "interleaved")
    att = lambda q, k, v: op.attention(q, k, v, Hq, Hkv, D, lens, 0.4)[0]
    for f, prim in ((rope, (rnd(N, (Hq + Hkv) * D), rnd(D), rnd(D))),
                    (att, (rnd(N, Hq * D), rnd(N, Hkv * D), rnd(N, Hkv * D)))):
        tang = tuple(rnd(*p.shape) for p in prim)
        y, yd = torch.func.jvp(f, prim, tang)
        assert (yd - _central(f, prim, tang)).abs().max() < 1e-8
        cot, dcot = rnd(*y.shape), rnd(*y.shape)
        gr, grd = op.grads_dual(f, prim, cot, tang, dcot)
        for i in range(3):
            num = _central(lambda c, *p: op.grads(f, p, c)[i], (cot,) + prim, (dcot,) + tang)
            assert (grd[i] - num).abs().max() < 1e-7
        # gradients against differences of the scalar <f, cot>
        for i in range(3):
            dirs = [torch.zeros_like(p) for p in prim]
            dirs[i] = rnd(*prim[i].shape)
            num = _central(lambda *p: (f(*p) * cot).sum(), prim, dirs)
            assert abs((gr[i] * dirs[i]).sum() - num) < 1e-7


def test_reference_bounds_cover_emulated_roundings():
    """The bounds of the GPU tests, against a CPU emulation that rounds the operands to bf16
    where the kernels do."""
    lens, Hq, Hkv, D = [40, 1, 23], 2, 1, 16
    v = au.data(lens, 0, Hq, Hkv, D, True, seed=3)
    ref, bound = au.reference(v, lens, Hq, Hkv, D)
    r16 = lambda t: t.bfloat16().double()
    a = 0
    for m in lens:
        s = slice(a, a + m)
        a += m
        for h in range(Hq):
            c = slice(h * D, (h + 1) * D)
            q, k, w = (v[n][s].double()[:, c if n == "q" else slice(0, D)] for n in ("q", "k", "v"))
            S = (q @ k.T * D ** -0.5).masked_fill(torch.ones(m, m, dtype=torch.bool).triu(1), -math.inf)
            e = torch.exp(S - S.amax(1, keepdim=True))
            o = r16((r16(e) @ w) / e.sum(1, keepdim=True))
            assert ((o - ref["o"][s, c]).abs() <= bound["o"][s, c]).all()
    assert all((b >= 0).all() for b in bound.values())
