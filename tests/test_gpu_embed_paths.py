"""Forms of the embedding gradient's kernels, each with sums that are held to that form's own depth: two
slabs a warp, ids whose tokens fill hundreds of blocks, sorts of four digits, one launch.

Depths.  A row's tokens are added one after the other inside a range of the path, then the ranges of a block,
then the blocks: by one warp where at most 31 blocks end inside the row, else by sixteen warps, a sixteenth of
the blocks each, and those sums.  A range has 64 steps at most and up to 31 tokens of the border behind it, a
block four ranges.  In the one launch a block has sixteen ranges of at most a sixteenth of the tokens and its
rows.  Every addition is off by 2^-24 of the magnitudes summed, and the scale and its product by as much."""
import ctypes as C
import math

import pytest

from gpu_util import need_gpu
from test_gpu_embed import CASES, U, make, reference, run

MARK = -7.0


def sorted_depth(torch, count):
    blocks = torch.ceil(count / (4 * 32)) + 1
    join = torch.maximum(blocks.clamp_max(31), torch.ceil(blocks / 16) + 16 * (blocks > 31))
    return count.clamp_max(64 + 31) + 4 + join + 1


def one_launch_depth(torch, count, n, vocab):
    return count.clamp_max(math.ceil((n + min(vocab, 8192)) / 16)) + 16


def check_depths(torch, native, s, n, scale, dual):
    o = run(torch, native, s, scale, dual)
    torch.cuda.synchronize()
    V, D = s["E"].shape
    one = native.mf_embed_work_bytes(len(s["ids"]), V, D, dual) == 16
    for t in ("", "d")[:1 + dual]:
        _, dE, size, count = reference(torch, s, n, scale, t)
        depth = one_launch_depth(torch, count, n, V) if one else sorted_depth(torch, count)
        depth = torch.minimum(depth, count + 1).unsqueeze(1)
        off = (o["dE" + t].double() - dE).abs()
        assert (off <= size * (depth + 3) * U + 2.0 ** -126).all(), ("dE" + t, (off / size).max().item() / U)
        assert (o["dE" + t][count == 0] == 0).all()
        wide = o["wide_dE" + t]
        assert (wide[:, :8] == MARK).all() and (wide[:, 8 + D:] == MARK).all()
    return o


@pytest.mark.gpu
@pytest.mark.parametrize("dual", [False, True])
@pytest.mark.parametrize("name", ["few", "odd_width", "slab", "past_slab", "one_row_table", "many_tiles", "long_tiles",
                                  "all_one_id", "heavy", "one_launch_tokens", "more_tokens", "all_one_id_long",
                                  "cluster_most", "launches_one_digit", "launches_three_digits"])
def test_depths(name, dual):
    torch, native = need_gpu()
    s = make(torch, CASES[name], 92, dual)
    check_depths(torch, native, s, CASES[name][0], 1.0, dual)


# bf16 rows, more than one slab, over 934000 steps and slabs: two slabs a warp
TWO_SLABS = {
    "odd_slabs": (200003, 5, 120001, 300, "f32", "bf16", "heavy", 0.1, False),
    "odd_slabs_tangents": (100001, 0, 60001, 300, "f32", "bf16", "heavy", 0.1, True),
    "last_column": (150000, 0, 90001, 385, "bf16", "bf16", "zipf", 0, False),
    "two_slabs_tangents": (200001, 40, 50007, 136, "f32", "bf16", "uniform", 0.2, True),
    "one_id": (260001, 0, 60000, 516, "f32", "bf16", "all", 0, False),
    "one_id_tangents": (330001, 0, 5000, 260, "f32", "bf16", "all", 0.3, True),
    "few_ids": (500001, 3, 7, 256, "f32", "bf16", "uniform", 0.01, False),
}


@pytest.mark.gpu
@pytest.mark.parametrize("name", list(TWO_SLABS))
def test_two_slabs_a_warp(name):
    torch, native = need_gpu()
    *case, dual = TWO_SLABS[name]
    N, tail, V, D = case[:4]
    slabs = -(-D // 128) * (1 + dual)
    assert (N + tail + V) // 64 * slabs >= 4 * 152 * 24 and D > 128
    s = make(torch, tuple(case), 93, dual)
    check_depths(torch, native, s, N, 1.0, dual)


@pytest.mark.gpu
@pytest.mark.parametrize("dual", [False, True])
@pytest.mark.parametrize("ty", ["f32", "bf16"])
def test_ids_of_thousands_of_blocks(ty, dual):
    """A row whose tokens lie in more blocks than the joining block has threads, beside others that do."""
    torch, native = need_gpu()
    s = make(torch, (400000, 0, 60, 9, "f32", ty, "all", 0.05), 94, dual)
    s["ids"][100000:170000], s["ids"][170000:200000] = 31, 29
    check_depths(torch, native, s, 400000, -0.5, dual)
    for t in ("", "d")[:1 + dual]:
        s["dy" + t].mul_(3).round_()
    o = run(torch, native, s, 2.0, dual)
    for t in ("", "d")[:1 + dual]:
        assert torch.equal(o["dE" + t].double(), reference(torch, s, 400000, 2.0, t)[1])


@pytest.mark.gpu
@pytest.mark.parametrize("n", [40, 20000, 40000])
@pytest.mark.parametrize("vocab", [2 ** 27 - 1, 2 ** 27, 2 ** 27 + 300])
def test_sorts_of_four_digits(n, vocab):
    """Tables of 2^27 rows and more (keys of 28 bits, the last for padding), one column."""
    torch, native = need_gpu()
    g = torch.Generator(device="cuda").manual_seed(95)
    ids = torch.randint(0, vocab, (n,), generator=g, device="cuda", dtype=torch.int64)
    ids[::3] = vocab - 1 - ids[::3] % 5
    ids[::7] = ids[::7] % 4 * 2 ** 25 + 77
    ids[::11] = vocab
    dy = torch.randint(-4, 5, (n, 8), generator=g, device="cuda").bfloat16()
    dE = torch.full((vocab, 8), MARK, device="cuda")
    work = torch.empty(native.mf_embed_work_bytes(n, vocab, 1), dtype=torch.uint8, device="cuda")
    native.mf_embed_bwd(ids.int(), dy[:, :1], dE[:, :1], work, scale=2.0)
    real = ids < vocab
    want = torch.zeros(vocab, dtype=torch.float32, device="cuda").index_add_(0, ids[real], 2 * dy[real, 0].float())
    assert torch.equal(dE[:, 0], want) and (dE[::1009, 1:] == MARK).all()
    E = torch.zeros(vocab, 8, device="cuda")
    E[:, 0] = torch.arange(vocab, device="cuda") % 8191
    y = torch.full((n, 8), MARK, device="cuda")
    native.mf_embed_fwd(ids.int(), E[:, :1], y[:, :1], scale=3.0)
    assert torch.equal(y[:, 0], torch.where(real, ids % 8191, 0).float() * 3) and (y[:, 1:] == MARK).all()
    del dE, E, want
    torch.cuda.empty_cache()


@pytest.mark.gpu
@pytest.mark.parametrize("vocab,dim", [(70, 20), (200000, 1024)])
def test_no_rows_with_the_args_of_the_call(vocab, dim):
    """The C call without rows: dE and dE' all zeros, from the workspace that the same args ask for."""
    torch, native = need_gpu()
    ld = -(-dim // 8) * 8
    dE, dEd = (torch.full((vocab, ld), MARK, device="cuda") for _ in range(2))
    a = native.mf_embed_args(n_rows=0, vocab=vocab, dim=dim, y_prec=1, scale=1.0, dE=dE.data_ptr(), dEd=dEd.data_ptr(), lddE=ld)
    size = C.c_size_t()
    assert native.lib().mf_embed_work_bytes(C.byref(a), C.byref(size)) == 0
    work = torch.empty(size.value, dtype=torch.uint8, device="cuda")
    a.work, a.work_bytes = work.data_ptr(), size.value
    assert native.lib().mf_embed_bwd(C.byref(a), None) == 0
    torch.cuda.synchronize()
    for t in (dE, dEd):
        assert (t[:, :dim] == 0).all() and (t[:, dim:] == MARK).all()
