"""The error bounds of the packed attention's GPU tests, without a GPU: an emulation that rounds to
bf16 where the kernels do stays inside them for every output, and mistakes do not."""
import pytest

import attn_rms_util as ar

SETS = {
    "ragged": ([300, 1, 77], 2, 1, 64, 0.0),
    "short": ([2] * 30 + [5, 3, 9, 1, 40], 4, 2, 32, 0.0),
    "one_token": ([1] * 20, 2, 1, 16, 0.0),
    "shifted_10": ([200, 90], 2, 1, 64, 10.0),
    "shifted_30": ([200, 90], 4, 2, 32, 30.0),
}




def _case(name):
    lens, Hq, Hkv, D, offset = SETS[name]
    return ar.shifted(lens, 0, Hq, Hkv, D, True, 3, offset), (lens, Hq, Hkv, D)


@pytest.mark.parametrize("name", list(SETS))
def test_emulated_roundings_stay_inside(name):
    v, shape = _case(name)
    r, bound = ar.bounds(v, *shape)
    _, var = ar.variances(v, *shape)
    e = ar.emulate(v, *shape)
    for k in r:
        assert ((e[k] - r[k]).abs() <= bound[k]).all(), k
    ar.check_norms(e, r, var, sum(shape[0]))


def test_rounding_before_centring_does_not():
    v, shape = _case("shifted_30")
    r, var = ar.variances(v, *shape)
    e = ar.emulate(v, *shape, centre=False)
    for k in ("od", "dqd", "dkd"):
        assert (e[k] - r[k]).norm() > ar.SLACK * var[k].sum().sqrt(), k


# P v' out of o', dS K' out of dq', dO O' out of D' (and so of dk'), P'^T dO out of dv'.  One-token
# sequences have dS = P' = 0; where keys have a common part, what that makes of D's rounding hides
# dS K'.
LEFT_OUT = [(n, t) for n in SETS for t in ("od", "dqd", "dkd", "dvd")
            if t == "od" or n != "one_token" and not (t == "dqd" and n.startswith("shifted"))]


@pytest.mark.parametrize("name,term", LEFT_OUT)
def test_a_term_left_out_does_not(name, term):
    v, shape = _case(name)
    r, bound = ar.bounds(v, *shape)
    _, var = ar.variances(v, *shape)
    off = (ar.emulate(v, *shape, drop=(term,))[term] - r[term]).abs()
    assert off.norm() > ar.SLACK * var[term].sum().sqrt()
    if not name.startswith("shifted"):
        assert (off > bound[term]).any()
