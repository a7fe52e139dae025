"""Windowed attention over 2^31 - 324 rows, more than which a chunk of query rows does not fit below
2^31: the same bits as the last rows by themselves."""
import pytest

from gpu_util import need_gpu


@pytest.mark.gpu
def test_window_of_the_most_rows():
    torch, native = need_gpu()
    if torch.cuda.mem_get_info()[0] < 215 << 30:
        pytest.skip("needs 215 GB of device memory")
    first, rows, D, window, sinks = 2 ** 31 - 2048, 1724, 8, 500, 2
    x = torch.zeros(first + rows, D, dtype=torch.bfloat16, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(72)
    x[first:] = torch.randn(rows, D, generator=g, device="cuda").bfloat16()
    outs = []
    for v, starts in ((x, [0, first, first + 1500, first + rows]), (x[first:], [0, 1500, rows])):
        n = v.shape[0]
        o, dq, dk, dv = (torch.empty(n, D, dtype=torch.bfloat16, device="cuda") for _ in range(4))
        lse = torch.empty(1, n, device="cuda")
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        work = torch.empty(native.mf_attn_window_work_bytes(n, 1, 1, D, window, sinks), dtype=torch.uint8, device="cuda")
        kw = dict(n_heads=1, n_kv_heads=1, head_dim=D, window=window, n_sink=sinks, status=status,
                  seq_start=torch.tensor(starts, dtype=torch.int32, device="cuda"))
        for t in (o, dq, dk, dv):
            t[n - rows:].fill_(-7.0)
        native.mf_attn_window_fwd(v, v, v, o, lse, **kw)
        native.mf_attn_window_bwd(v, v, v, o, lse, v, dq, dk, dv, work=work, **kw)
        torch.cuda.synchronize()
        assert int(status.item()) == 0
        outs.append([t[n - rows:].clone() for t in (o, dq, dk, dv)] + [lse[:, n - rows:].clone()])
        # zeros attend to zeros
        assert (o[:1000] == 0).all() or n == rows
        del o, dq, dk, dv, lse, work
        torch.cuda.empty_cache()
    del x
    torch.cuda.empty_cache()
    for a, b in zip(*outs):
        assert torch.equal(a, b) and torch.isfinite(b).all() and not (b == -7.0).all()
