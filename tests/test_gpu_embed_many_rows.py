"""The largest number of rows: the gradient of an embedding and the lookup of 2^31 - 257 tokens, nearly
all of them padding.  Whole numbers, so that sums are exact."""
import pytest

from gpu_util import need_gpu


@pytest.mark.gpu
@pytest.mark.parametrize("n", [2 ** 31 - 257, 2 ** 31 - 4096])
def test_embed_of_the_most_rows(n):
    torch, native = need_gpu()
    V = 700
    if torch.cuda.mem_get_info()[0] < 120 << 30:
        pytest.skip("needs 120 GB of device memory")
    ids = torch.full((n,), -1, dtype=torch.int32, device="cuda")
    wide = torch.empty(n, 8, dtype=torch.bfloat16, device="cuda")       # padding's rows hold anything
    tile = 2 ** 25                    # of a block of the sort
    at = [0, 1, tile - 1, tile, 2 ** 30, 63 * tile - 1, 63 * tile, 2 ** 31 - 8192, 2 ** 31 - 4097, n - 1]
    at = torch.tensor(sorted({i for i in at if i < n}) + list(range(10 ** 9, 10 ** 9 + 5000)), device="cuda")
    g = torch.Generator(device="cuda").manual_seed(90)
    tokens = torch.randint(0, V, (len(at),), device="cuda", generator=g)
    rows = torch.randint(-4, 5, (len(at),), device="cuda", generator=g)
    ids[at], wide[at, 0] = tokens.int(), rows.bfloat16()
    dE = torch.full((V, 8), -7.0, device="cuda")
    work = torch.empty(native.mf_embed_work_bytes(n, V, 1), dtype=torch.uint8, device="cuda")
    native.mf_embed_bwd(ids, wide[:, :1], dE[:, :1], work, scale=2.0)
    want = torch.zeros(V, dtype=torch.float64, device="cuda").index_add_(0, tokens, 2.0 * rows.double())
    assert torch.equal(dE[:, 0].double(), want)
    del work
    E = torch.randint(1, 60, (V, 8), device="cuda", generator=g).float()
    wide[at, 1] = -7.0
    native.mf_embed_fwd(ids, E[:, :1], wide[:, :1], scale=2.0)
    assert torch.equal(wide[at, 0].float(), 2.0 * E[tokens, 0]) and (wide[at, 1] == -7.0).all()
    pads = torch.cat([torch.arange(n - 4000, n, device="cuda"), torch.randint(0, n, (10 ** 6,), device="cuda", generator=g)])
    pads = pads[ids[pads] < 0]
    assert len(pads) > 10 ** 5 and (wide[pads, 0] == 0).all()
    del ids, wide
    torch.cuda.empty_cache()
