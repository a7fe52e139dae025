"""Decoders with grouped heads, head norms and rotary variants (mf_create_decoder) through the
C ABI against the float64 oracle.

The bound is that of the other bf16 decoders, 2e-2 in relative L2: the same tensors are rounded
to bf16, and with them dO and dq, dk, dv before the inverse rotation, each by 2^-8 of the value
at most, which adds at most 4 * 2^-8 = 1.6e-2 in the worst case and, the roundings of single
elements being independent, far less in the norm of a sum over hundreds of them."""
import math

import numpy as np
import pytest

from gpu_util import need_gpu, rel_l2
from paper_2505_00793_gb300 import synth
from oracle import metagrad as om
from test_gpu_decoder import _run

EX, SLR, PLR = synth.EXAMPLE_WEIGHTS, synth.SCALAR_LOGLR, synth.PARAM_LOGLR
TOL = 2e-2

CASES = {
    # four heads over two, norms; a sequence of half a tile
    "grouped_norm": synth.decoder("grouped_norm", 128, 4, 256, 2, 256, 64, B=4, T=2, B_outer=3,
                                  alpha=1e-2, n_kv_heads=2, qk_norm=True),
    # one key/value head, part of each head turned pair by pair, tiles that hold several sequences
    "one_kv": synth.decoder("one_kv", 128, 2, 128, 1, 200, 40, B=5, T=2, B_outer=2, momentum=0.9,
                            meta_kind=EX | SLR, extra={"scalar_loglr": math.log(1e-2)},
                            n_kv_heads=1, rope={"layout": "interleaved", "dims": 32}),
    # norms without groups, stretched positions, learning rates of the gains among the others
    "norm_bands": synth.decoder("norm_bands", 96, 4, 128, 2, 128, 136, B=2, T=2, B_outer=2,
                                meta_kind=EX | PLR, loglr_mean=math.log(1e-2), loglr_std=0.1,
                                qk_norm=True, rope={"scaling": "bands", "factor": 4.0,
                                                    "orig_len": 64}),
}


def _inputs(w):
    """Inputs whose head gains differ from one another."""
    inp, o = synth.make_inputs(w), 0
    for name, n in w.decoder_layout():
        if name[:2] in ("gq", "gk"):
            inp.theta0[o:o + n] += 0.2 * synth.random_direction(n, 5, o % 97)
        o += n
    return inp


@pytest.mark.parametrize("name", list(CASES))
def test_layout(name):
    """The flat vector is as long as the tensors, and the gains lie on 16-byte boundaries."""
    w, o = CASES[name], 0
    for t, n in w.decoder_layout():
        assert o % 4 == 0, t
        o += n
    assert o == w.n_params


def test_oracle_agrees_with_plain_heads():
    """Without groups, norms or scaling the packed attention is the plain decoder's."""
    import torch
    from oracle import model
    w = synth.decoder("p", 32, 2, 48, 2, 40, 16, B=2, T=1, B_outer=1)
    inp = synth.make_inputs(w)
    th = torch.from_numpy(inp.theta0.astype(np.float64))
    ids = torch.from_numpy(inp.inner_x[0]).long()
    a, b = (model.decoder_losses(v, th, ids) for v in (w, w.with_(rope={})))
    assert torch.allclose(a, b, rtol=1e-12, atol=0)


def test_refusals():
    """Bad heads are refused before the device is looked at."""
    import ctypes as C
    from paper_2505_00793_gb300 import build, native
    build.build()
    lib, h = native.load(), C.c_void_p()

    def create(kv=0, norm=0, rope=None, **kw):
        w = CASES["grouped_norm"].with_(**kw)
        d = native.model_desc_for(w)
        heads = native.mf_decoder_heads(kv, norm, native.rope_desc(**(rope or {})))
        return lib.mf_create_decoder(C.byref(d), C.byref(heads), C.byref(h))

    assert lib.mf_create_decoder(None, None, C.byref(h)) == 1
    assert create(kv=3) == 1 and create(kv=-1) == 1 and create(kv=8) == 1
    assert create(norm=2) == 1
    assert create(rope={"dims": 34}) == 1 and create(rope={"dims": 7}) == 1
    assert create(rope={"base": -1.0}) == 1 and create(rope={"scaling": "linear", "factor": 0.0}) == 1
    assert create(precision="fp32") == 2
    assert create(d_model=512) == 2                       # heads of 128
    assert create(d_model=1024) == 1                      # of 256
    d = native.model_desc_for(synth.WORKLOADS["wide"])    # no decoder
    assert lib.mf_create_decoder(C.byref(d), C.byref(native.mf_decoder_heads()), C.byref(h)) == 1


@pytest.mark.gpu
@pytest.mark.parametrize("name", list(CASES))
def test_meta_grad(name):
    w = CASES[name]
    inp = _inputs(w)
    ref, got = om.meta_grad(w, inp), _run(w, inp)
    assert abs(got["V"] - ref["V"]) <= TOL * abs(ref["V"])
    assert rel_l2(got["d_theta0"], ref["d_theta0"]) < TOL
    assert rel_l2(got["d_eta"], ref["d_eta"]) < TOL


@pytest.mark.gpu
@pytest.mark.parametrize("mode", ["mixed", "rev_rev"])
@pytest.mark.parametrize("name", list(CASES))
def test_hvp(name, mode):
    """Gradient, H v and tangent losses, the gains' own parts among them."""
    torch, native = need_gpu()
    w = CASES[name]
    inp = _inputs(w)
    ids = inp.inner_x[0]
    v = synth.random_direction(w.n_params, 2, 3)
    wt = np.linspace(0.3, 1.0, w.B).astype(np.float32)
    mf = native.MixFlow.for_workload(w)
    assert mf.param_count()[0] == w.n_params
    d = native.to_device_inputs(w, inp)
    Hv = torch.full((w.n_params,), float("nan"), device="cuda")
    g = torch.full((w.n_params,), float("nan"), device="cuda") if mode == "mixed" else None
    tl = torch.full((w.B,), float("nan"), device="cuda")
    mf.hvp(w.B, d["theta0"], d["inner_x"][0], d["inner_y"][0], torch.from_numpy(v).cuda(), Hv,
           ex_w=torch.from_numpy(wt).cuda(), tangent_losses=tl, grad=g,
           hvp_mode=native.MF_HVP_REV_REV if mode == "rev_rev" else native.MF_HVP_MIXED_FOR)
    mf.sync()
    ref = om.hvp(w, inp.theta0, ids, ids, v, wt)
    Hv = Hv.cpu().numpy()
    assert rel_l2(Hv, ref) < TOL
    assert rel_l2(tl.cpu().numpy(), om.tangent_losses(w, inp.theta0, ids, ids, v)) < TOL
    if g is not None:
        assert rel_l2(g.cpu().numpy(), om.grad(w, inp.theta0, ids, ids, wt)) < TOL
    if w.qk_norm:
        own, o = [], 0
        for t, n in w.decoder_layout():
            if t[:2] in ("gq", "gk"):
                own.append(slice(o, o + n))
            o += n
        own = np.r_[tuple(own)]
        assert rel_l2(Hv[own], ref[own]) < TOL
    mf.close()


@pytest.mark.gpu
def test_same_bits_with_every_option():
    """Graphs, the side stream, early launches and checkpoints do not change a bit."""
    torch, native = need_gpu()
    w = CASES["grouped_norm"].with_(T=3)
    inp = _inputs(w)
    d = native.to_device_inputs(w, inp)
    outs, defaults = [], {native.MF_OPT_CUDA_GRAPHS: 1, native.MF_OPT_CONCURRENT: 1, native.MF_OPT_PDL: 1}
    mf = native.MixFlow.for_workload(w)
    try:
        for opts, every in (({}, 1), ({native.MF_OPT_CUDA_GRAPHS: 0}, 1), ({native.MF_OPT_CONCURRENT: 0}, 1),
                            ({native.MF_OPT_PDL: 0}, 1), ({}, 2)):
            for k, v in {**defaults, **opts}.items():
                mf.set_option(k, v)
            loop = native.loop_desc_for(w, ckpt_every=every)
            for _ in range(2):
                d_eta = torch.full((w.n_eta,), float("nan"), device="cuda")
                d_th = torch.full((w.n_params,), float("nan"), device="cuda")
                mf.meta_grad(loop, d["theta0"], d["eta"], d["inner_x"], d["inner_y"], d["outer_x"],
                             d["outer_y"], d_eta, d_th, None)
                mf.sync()
                outs.append((d_eta.clone(), d_th.clone()))
    finally:
        for k, v in defaults.items():    # early launches are the process's own switch
            mf.set_option(k, v)
        mf.close()
    for a, b in outs[1:]:
        assert torch.equal(a, outs[0][0]) and torch.equal(b, outs[0][1])
