"""Calls of the operators on packed token rows that the documentation allows, and what a decoder
handle made of them reserves."""
import pytest

import attn_ops_util as au
from gpu_util import need_gpu
from paper_2505_00793_gb300 import synth


@pytest.mark.gpu
@pytest.mark.parametrize("D,dual", [(64, False), (64, True), (128, False), (24, True)])
@pytest.mark.parametrize("n,length", [(1, 300), (300, 1), (5, 60), (2, 128), (3, 129)])
def test_equal_sequences_by_their_number(D, dual, n, length):
    torch, native = need_gpu()
    Hq, Hkv, N = 4, 2, n * length
    v = au.wide(au.data([length] * n, 0, Hq, Hkv, D, dual, seed=51))
    want = au.run(native, v, [length] * n, Hq, Hkv, D)
    out = {k: (torch.full_like(t, au.MARK) if k in au.names(dual) else t.clone()) for k, t in want.items()}
    t = lambda *names: {k: out[k] for k in names} if dual else {}
    kw = dict(n_heads=Hq, n_kv_heads=Hkv, head_dim=D, status=out["status"], n_seq=n,
              **{k: v[k] for k in ("qd", "kd", "vd") if dual}, **t("od", "rbar"))
    native.mf_attn_fwd(v["q"], v["k"], v["v"], out["o"], out["lse"], **kw)
    native.mf_attn_bwd(v["q"], v["k"], v["v"], out["o"], out["lse"], v["do"], out["dq"], out["dk"],
                       out["dv"], work=out["work"], dod=v.get("dod"), **t("dqd", "dkd", "dvd"), **kw)
    torch.cuda.synchronize()
    assert int(out["status"].item()) == 0
    for k in au.names(dual):
        assert torch.equal(out[k], want[k]), k
    assert N == out["o"].shape[0]


@pytest.mark.gpu
def test_rope_primal_backward_beside_a_tangent():
    """xd given, no tangent of dy: the gradients of the primal pass, in its workspace."""
    torch, native = need_gpu()
    N, Hq, Hkv, D = 70, 3, 1, 64
    g = torch.Generator().manual_seed(52)
    rnd = lambda *s: torch.randn(*s, generator=g).cuda()
    W = (Hq + Hkv) * D
    x, xd, dy, gq, gk = rnd(N, W), rnd(N, W), rnd(N, W), rnd(D), rnd(D)
    kw = dict(n_heads=Hq, n_kv_heads=Hkv, head_dim=D, rope=native.rope_desc(), gq=gq, gk=gk)
    work = torch.empty(native.mf_qk_rope_work_bytes(N, Hq, Hkv, D), dtype=torch.uint8, device="cuda")
    got = []
    for tangent in (None, xd):
        o = [torch.full_like(x, 3.0), torch.empty(D, device="cuda"), torch.empty(D, device="cuda")]
        native.mf_qk_rope_bwd(dy, o[0], x=x, xd=tangent, dgq=o[1], dgk=o[2], work=work, **kw)
        got.append(o)
    torch.cuda.synchronize()
    for a, b in zip(*got):
        assert torch.equal(a, b)


@pytest.mark.gpu
def test_norms_reserve_what_they_use():
    """Head norms keep each block's projected rows and their tangents, in place of the one pair of
    buffers that all blocks share without norms."""
    torch, native = need_gpu()
    w = synth.decoder("ws", 128, 4, 256, 2, 256, 128, B=16, T=2, B_outer=16, n_kv_heads=2, qk_norm=True)
    size = {}
    for norm in (True, False):
        v = w.with_(qk_norm=norm)
        mf = native.MixFlow.for_workload(v)
        size[norm] = mf.workspace_bytes(native.loop_desc_for(v))
        mf.close()
    pair = 2 * 16 * 128 * (4 + 2 * 2) * 32 * 4
    # the gains themselves, their copies and the workspace of their sums are below a quarter of it
    assert size[True] - size[False] <= (w.n_blocks - 1) * pair + pair // 4


@pytest.mark.gpu
def test_more_row_tiles_than_a_grid_is_high():
    """Tiles behind the 65535th: the same bits as those rows by themselves."""
    torch, native = need_gpu()
    D, L, n = 8, 64, 65535 * 128 + 384
    g = torch.Generator(device="cuda").manual_seed(53)
    v = {k: torch.randn(n, D, generator=g, device="cuda").bfloat16()
         for k in ("q", "k", "v", "do", "qd", "kd", "vd", "dod")}
    outs = []
    for rows in (n, 512):
        w = {k: t[n - rows:] for k, t in v.items()}
        starts = torch.arange(0, rows + 1, L, dtype=torch.int32, device="cuda")
        outs.append(au.run(native, w, None, 1, 1, D, starts=starts))
    torch.cuda.synchronize()
    assert int(outs[0]["status"].item()) == 0
    for k in au.names(True):
        a, b = outs[0][k], outs[1][k]
        a = a[:, n - 512:] if k in ("lse", "rbar") else a[n - 512:]
        assert torch.equal(a, b) and torch.isfinite(b).all(), k
        assert not (outs[0][k] == au.MARK).all(), k


@pytest.mark.gpu
@pytest.mark.parametrize("dual", [False, True])
def test_many_heads_of_few_rows(dual):
    """Two thousand query heads over one key head of eight columns."""
    torch, native = need_gpu()
    lens, Hq, Hkv, D = [3, 0, 5, 1], 2048, 1, 8
    v = au.data(lens, 2, Hq, Hkv, D, dual, seed=54)
    ref, bound = au.reference(v, lens, Hq, Hkv, D)
    out = au.run(native, au.wide(v), lens, Hq, Hkv, D)
    torch.cuda.synchronize()
    au.check(out, ref, bound, sum(lens), dual)


@pytest.mark.gpu
@pytest.mark.parametrize("D,dual", [(64, False), (64, True), (128, False)])
def test_sequences_do_not_feel_one_another(D, dual):
    """A sequence's bits do not depend on what shares its tiles: other sequences' maxima that move,
    tangents of other sizes, values near the largest."""
    torch, native = need_gpu()
    lens, Hq, Hkv = [40, 77, 200, 3, 130, 60], 4, 2
    v = au.data(lens, 9, Hq, Hkv, D, dual, seed=55)
    want = {k: t.clone() for k, t in au.run(native, au.wide(v), lens, Hq, Hkv, D).items()}
    others = [r for r in range(sum(lens) + 9) if not (117 <= r < 317 or 320 <= r < 450)]
    mine = [r for r in range(sum(lens)) if r not in others]
    for scale in (30.0, 1e-3, 1e18):
        w = {k: t.clone() for k, t in v.items()}
        for t in w.values():
            t[others] = (t[others].float() * scale).bfloat16()
        got = au.run(native, au.wide(w), lens, Hq, Hkv, D)
        torch.cuda.synchronize()
        for k in au.names(dual):
            a, b = (got[k].t(), want[k].t()) if k in ("lse", "rbar") else (got[k], want[k])
            assert torch.equal(a[mine], b[mine]), (scale, k)
