"""Every function of the library has its argument types declared: without them ctypes passes a Python
integer as a C int, and a stream's handle, a pointer, loses its upper half."""
import ctypes as C


def test_every_call_declares_its_arguments():
    from paper_2505_00793_gb300 import build, native
    build.build()
    L = native.load()
    for name in native.EXPORTS:
        assert getattr(L, name).argtypes is not None, name
    for op in ("mf_qk_rope", "mf_attn", "mf_attn_window", "mf_embed"):
        for call in ("fwd", "bwd", "work_bytes"):
            assert getattr(L, f"{op}_{call}").argtypes[-1] is C.c_void_p
