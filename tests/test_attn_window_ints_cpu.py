"""Windows and sinks beyond the C types keep their meaning through the binding."""
import pytest


@pytest.fixture(scope="module")
def native():
    from paper_2505_00793_gb300 import build, native
    build.build()
    return native


def test_integers_beyond_the_c_types(native):
    f = native.mf_attn_window_work_bytes
    every = native.mf_attn_work_bytes(512, 4)
    assert f(512, 4, 2, 64, 4, 0) == every
    rows = f(2000, 4, 2, 64, 2000, 5)
    for window in (2 ** 63 - 1, 2 ** 63, 2 ** 64 + 4, 10 ** 30):
        assert f(2000, 4, 2, 64, window, 5) == rows
    for window, sinks, status in ((-2 ** 63 - 5, 5, 1), (-2 ** 64 + 4, 5, 1), (4, -2 ** 32 + 5, 1), (4, -10 ** 20, 1),
                                  (4, 2 ** 32 + 5, 2), (4, 2 ** 31, 2), (4, 10 ** 20, 2), (4, 129, 2)):
        with pytest.raises(native.MixflowError) as e:
            f(2000, 4, 2, 64, window, sinks)
        assert e.value.status == status, (window, sinks)
