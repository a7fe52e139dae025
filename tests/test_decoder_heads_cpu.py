"""mf_create_decoder refuses at once what its first call would refuse, without a GPU."""
import ctypes as C
import math

import pytest

from paper_2505_00793_gb300 import synth


@pytest.fixture(scope="module")
def native():
    from paper_2505_00793_gb300 import build, native
    build.build()
    return native


def _create(native, norm=True, rope=None, **kw):
    w = synth.decoder("d", 128, 4, 256, 2, 256, 64, B=4, T=2, B_outer=3, alpha=1e-2).with_(**kw)
    d, h = native.model_desc_for(w), C.c_void_p()
    heads = native.mf_decoder_heads(2, int(norm), native.rope_desc(**(rope or {})))
    return native.load().mf_create_decoder(C.byref(d), C.byref(heads), C.byref(h))


@pytest.mark.parametrize("rope", [{"base": 0.0}, {"base": 0.0, "scaling": "linear", "factor": 2.0}], ids=str)
def test_base_taken_from_the_model(native, rope):
    assert _create(native, rope=rope, rope_base=math.inf) == 1


def test_eps_of_the_norms(native):
    assert _create(native, rms_eps=math.inf) == 1


@pytest.mark.parametrize("rope", [{"base": math.inf}, {"base": math.nan}, {"mscale": math.inf}], ids=str)
def test_own_rotary_positions(native, rope):
    assert _create(native, rope=rope) == 1
