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
