"""Embedding lookup with scaling and its gradient (mf_embed_fwd / mf_embed_bwd) against the float64
definition: every type pair, tables and widths around every edge of the sort and of the sums' ranges,
one id for all tokens, padding, rows behind the last sequence, strided rows, values that are not
finite, streams, graphs.

Bounds.  A lookup is one float32 product (2^-24 of it, and as much again for the scale's own rounding)
rounded to its type.  A gradient passes through at most 512 + 32 additions of a range, then those of a
block's ranges and of the blocks that share the row: below 1100 in all for up to 2^18 tokens, and never
more than its tokens and eight; each is off by 2^-24 of the magnitudes summed."""
import math

import pytest

from gpu_util import need_gpu

MARK = -7.0
U = 2.0 ** -24
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}

CASES = {
    # rows, tail, vocab, dim, table type, row type, ids, share of padding
    "one": (1, 0, 1, 1, "f32", "f32", "zipf", 0),
    "few": (7, 0, 50, 16, "f32", "f32", "zipf", 0),
    "odd_width": (33, 3, 12, 5, "bf16", "f32", "uniform", 0.2),
    "slab": (300, 0, 40, 128, "f32", "bf16", "zipf", 0.1),
    "past_slab": (300, 9, 40, 129, "bf16", "bf16", "zipf", 0.1),
    "below_slab": (200, 0, 500, 127, "bf16", "f32", "uniform", 0),
    "wide": (100, 1, 30, 1500, "f32", "f32", "zipf", 0),
    "very_wide": (9, 0, 5, 5001, "bf16", "bf16", "uniform", 0),
    "one_row_table": (1000, 0, 1, 24, "f32", "bf16", "uniform", 0.3),
    "one_digit": (5000, 7, 510, 40, "f32", "f32", "zipf", 0),
    "two_digits": (5000, 0, 511, 40, "f32", "f32", "uniform", 0),
    "three_digits": (4097, 0, 2 ** 18, 8, "f32", "f32", "zipf", 0.05),
    "sort_tile": (4096, 0, 3000, 36, "f32", "bf16", "uniform", 0),
    "many_tiles": (40001, 20, 20000, 12, "f32", "f32", "zipf", 0.1),
    "long_tiles": (2 ** 18 + 77, 0, 1000, 4, "f32", "f32", "zipf", 0),
    "all_one_id": (3000, 0, 700, 130, "f32", "f32", "all", 0),
    "border": (32, 0, 40, 8, "f32", "f32", "all", 0),
    "heavy": (20000, 0, 5000, 200, "f32", "bf16", "heavy", 0.1),
    "last_id": (500, 0, 900, 20, "f32", "f32", "last", 0),
    # the most tokens and the most rows of one launch, and one more
    "one_launch_tokens": (6144, 0, 3000, 24, "f32", "bf16", "heavy", 0.1),
    "more_tokens": (6145, 0, 3000, 24, "f32", "bf16", "heavy", 0.1),
    "one_launch_rows": (40, 0, 304 * 8192, 3, "f32", "f32", "uniform", 0),
    "more_rows": (40, 0, 304 * 8192 + 1, 3, "f32", "f32", "uniform", 0),
    "one_block": (700, 3, 9, 7, "f32", "bf16", "zipf", 0.1),
    "one_block_a_part": (500, 0, 8192, 40000, "bf16", "bf16", "heavy", 0),
    "all_one_id_long": (9000, 0, 700, 130, "f32", "f32", "all", 0),
    "border_long": (32, 0, 304 * 8192 + 1, 8, "f32", "f32", "all", 0),
    # sorts of one, two and three digits, by one cluster and by launches
    "cluster_one_digit": (7000, 7, 510, 40, "f32", "f32", "zipf", 0),
    "cluster_two_digits": (8192, 0, 511, 40, "f32", "bf16", "uniform", 0),
    "cluster_three_digits": (9001, 0, 2 ** 18, 8, "f32", "f32", "zipf", 0.05),
    "cluster_most": (32768, 0, 3000, 12, "f32", "f32", "zipf", 0.1),
    "launches_one_digit": (32769, 0, 200, 12, "f32", "f32", "uniform", 0.1),
    "launches_three_digits": (33000, 9, 300000, 4, "f32", "bf16", "zipf", 0.1),
    "padding_only": (400, 5, 100, 64, "f32", "f32", "zipf", 1),
}


def make(torch, case, seed, dual):
    N, tail, V, D, te, ty, kind, pad = case
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt = {"f32": torch.float32, "bf16": torch.bfloat16}
    rnd = lambda *s: torch.randn(*s, device="cuda", generator=g)
    rand = lambda: torch.rand(N + tail, device="cuda", generator=g, dtype=torch.float64)
    ids = (rand() * V).long() if kind == "uniform" else (torch.exp(rand() * math.log(V + 1.0)) - 1).long()
    if kind == "heavy":
        ids[rand() < 0.4] = V // 3
    if kind in ("all", "last"):
        ids[:] = V - 1 if kind == "last" else V // 2
    ids = ids.clamp(0, V - 1)
    out = rand() < pad
    ids[out] = torch.where(rand() < 0.5, -1 - ids, V + ids)[out]      # outside on both sides
    ids[N:] = torch.arange(tail, device="cuda") * 10 ** 8 - 5
    s = {"ids": ids.int(), "start": torch.tensor([0, N // 3, N], dtype=torch.int32, device="cuda")}
    for t in ("", "d")[:1 + dual]:
        s["E" + t], s["dy" + t] = strided(torch, rnd(V, D).to(dt[te])), strided(torch, rnd(N + tail, D).to(dt[ty]))
    return s


def rows(torch, n, D, dtype, value=MARK):
    """A column range of wider rows that begins and ends inside them, and all of the rows."""
    w = torch.full((n, -(-D // 8) * 8 + 16), value, dtype=dtype, device="cuda")
    return w[:, 8:8 + D], w


def strided(torch, t):
    x, _ = rows(torch, *t.shape, t.dtype, math.nan)
    x.copy_(t)
    return x


def run(torch, native, s, scale, dual, stream=None, start=True, out=None):
    N, (V, D) = len(s["ids"]), s["E"].shape
    o = out or {}
    if not out:
        for t in ("", "d")[:1 + dual]:
            o["y" + t], o["wide_y" + t] = rows(torch, N, D, s["dy"].dtype)
            o["dE" + t], o["wide_dE" + t] = rows(torch, V, D, torch.float32)
        o["work"] = torch.full((native.mf_embed_work_bytes(N, V, D, dual),), 255, dtype=torch.uint8, device="cuda")
    kw = dict(scale=scale, seq_start=s["start"] if start else None, stream=stream)
    native.mf_embed_fwd(s["ids"], s["E"], o["y"], Ed=s.get("Ed"), yd=o.get("yd"), **kw)
    native.mf_embed_bwd(s["ids"], s["dy"], o["dE"], o["work"], dyd=s.get("dyd"), dEd=o.get("dEd"), **kw)
    return o


def reference(torch, s, n, scale, t):
    """(y, dE, magnitudes summed, tokens) in float64."""
    V, D = s["E"].shape
    ids = s["ids"][:n].long()
    real = (ids >= 0) & (ids < V)
    E, dy = s["E" + t].double(), s["dy" + t][:n].double()
    y = E[ids.clamp(0, V - 1)] * (real * scale).unsqueeze(1)
    dE, size = (torch.zeros(V, D, dtype=torch.float64, device="cuda") for _ in range(2))
    dE.index_add_(0, ids[real], dy[real])
    size.index_add_(0, ids[real], dy[real].abs())
    count = torch.zeros(V, dtype=torch.float64, device="cuda").index_add_(0, ids[real], torch.ones_like(dy[real][:, 0]))
    return y, dE * scale, size * abs(scale), count


def check(torch, o, s, n, scale, dual, ty):
    f32 = torch.tensor(scale, dtype=torch.float32).item()
    for t in ("", "d")[:1 + dual]:
        y, dE, size, count = reference(torch, s, n, scale, t)
        got = o["y" + t]
        assert ((got[:n].double() - y).abs() <= y.abs() * (HALF[ty] + 3 * U) + 2.0 ** -126).all(), "y" + t
        assert (got[n:] == MARK).all()
        depth = (count + 8).clamp_max(1100).unsqueeze(1)
        off = (o["dE" + t].double() - dE).abs()
        assert (off <= size * (depth + 3) * U + 2.0 ** -126).all(), ("dE" + t, off.max().item())
        assert (o["dE" + t][count == 0] == 0).all()
        # what lies beside the columns stays
        for name in ("wide_y" + t, "wide_dE" + t):
            if name in o:
                assert (o[name][:, :8] == MARK).all() and (o[name][:, 8 + s["E"].shape[1]:] == MARK).all(), name
    assert math.isfinite(f32)


@pytest.mark.gpu
@pytest.mark.parametrize("dual", [False, True])
@pytest.mark.parametrize("name", list(CASES))
def test_embed_against_definition(name, dual):
    torch, native = need_gpu()
    case = CASES[name]
    s = make(torch, case, 81, dual)
    scale = 27.7 if dual else 0.3
    o = run(torch, native, s, scale, dual)
    torch.cuda.synchronize()
    check(torch, o, s, case[0], scale, dual, case[5])


@pytest.mark.gpu
@pytest.mark.parametrize("te", ["f32", "bf16"])
@pytest.mark.parametrize("ty", ["f32", "bf16"])
def test_embed_types(te, ty):
    torch, native = need_gpu()
    case = (333, 4, 90, 52, te, ty, "zipf", 0.1)
    s = make(torch, case, 82, True)
    o = run(torch, native, s, -1.5, True)
    torch.cuda.synchronize()
    check(torch, o, s, 333, -1.5, True, ty)


@pytest.mark.gpu
@pytest.mark.parametrize("name", ["two_digits", "many_tiles", "all_one_id", "heavy", "long_tiles", "more_tokens", "one_launch_tokens",
                                  "all_one_id_long", "cluster_one_digit", "cluster_most", "launches_one_digit",
                                  "launches_three_digits"])
def test_embed_whole_numbers_are_exact(name):
    """Small whole numbers sum exactly in any order: every token once, in its own row."""
    torch, native = need_gpu()
    N, tail, V, D, _, _, kind, pad = CASES[name]
    s = make(torch, (N, tail, V, D, "f32", "f32", kind, pad), 83, True)
    for t in ("", "d"):
        s["dy" + t].mul_(3).round_()
    o = run(torch, native, s, 2.0, True)
    torch.cuda.synchronize()
    for t in ("", "d"):
        _, dE, _, _ = reference(torch, s, N, 2.0, t)
        assert torch.equal(o["dE" + t].double(), dE)


@pytest.mark.gpu
def test_embed_no_rows():
    """No tokens: a lookup that touches nothing, a gradient of zeros."""
    torch, native = need_gpu()
    for N, tail in ((0, 0), (0, 90)):
        s = make(torch, (N, tail, 70, 20, "f32", "f32", "zipf", 0), 84, True)
        o = run(torch, native, s, 1.0, True)
        torch.cuda.synchronize()
        for t in ("", "d"):
            assert (o["y" + t] == MARK).all() and (o["dE" + t] == 0).all()


@pytest.mark.gpu
def test_embed_all_rows_without_sequences():
    torch, native = need_gpu()
    s = make(torch, (500, 0, 60, 32, "f32", "bf16", "zipf", 0.1), 85, False)
    a, b = run(torch, native, s, 1.0, False), run(torch, native, s, 1.0, False, start=False)
    for k in ("y", "dE"):
        assert torch.equal(a[k], b[k])


@pytest.mark.gpu
@pytest.mark.parametrize("value", [math.nan, math.inf])
@pytest.mark.parametrize("tokens", [600, 8000])
def test_embed_values_that_are_not_finite(value, tokens):
    """A table row reaches the rows of its id alone, a row's gradient its id's row alone; padding and
    rows behind the last sequence reach nothing."""
    torch, native = need_gpu()
    case = (tokens, 30, 800, 72, "f32", "f32", "heavy", 0.1)
    s = make(torch, case, 86, False)
    want = {k: t.clone() for k, t in run(torch, native, s, 2.0, False).items()}
    ids = s["ids"][:tokens].long()
    pads = torch.nonzero((ids < 0) | (ids >= 800)).squeeze(1)
    s["dy"][pads] = value
    s["dy"][tokens:] = value
    row = torch.nonzero((ids >= 0) & (ids < 800))[17].item()
    s["dy"][row, 3] = value
    s["E"][5] = value
    o = run(torch, native, s, 2.0, False)
    torch.cuda.synchronize()
    keep = torch.ones_like(o["dE"], dtype=torch.bool)
    keep[ids[row], 3] = False
    assert torch.equal(o["dE"][keep], want["dE"][keep]) and not torch.isfinite(o["dE"][ids[row], 3])
    keep = s["ids"] != 5
    assert torch.equal(o["y"][keep], want["y"][keep]) and not torch.isfinite(o["y"][:tokens][ids == 5]).any()


@pytest.mark.gpu
def test_embed_same_bits_again_and_at_once():
    torch, native = need_gpu()
    jobs = []
    for seed, name in ((1, "many_tiles"), (2, "heavy"), (3, "slab"), (4, "one_launch_tokens")):
        s = make(torch, CASES[name], seed, True)
        jobs.append((s, {k: t.clone() for k, t in run(torch, native, s, 3.0, True).items()}))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in jobs]
    for _ in range(10):
        outs = []
        for (s, _), st in zip(jobs, streams):
            with torch.cuda.stream(st):
                outs.append(run(torch, native, s, 3.0, True))
        side = run(torch, native, jobs[0][0], 3.0, True, stream=torch.cuda.current_stream())
        torch.cuda.synchronize()
        for (_, want), got in zip(jobs + jobs[:1], outs + [side]):
            for k in ("y", "yd", "dE", "dEd"):
                assert torch.equal(got[k], want[k]), k


@pytest.mark.gpu
@pytest.mark.parametrize("rows", [6000, 9000, 40000])
def test_embed_captured_with_other_tokens(rows):
    """A captured call replayed after ids, lengths and gradients have changed on the device."""
    torch, native = need_gpu()
    N, V, D = rows, 2000, 48
    s = make(torch, (N, 0, V, D, "f32", "f32", "zipf", 0.1), 87, True)
    o = run(torch, native, s, 1.5, True)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        run(torch, native, s, 1.5, True, out=o)
    for seed, kind, n in ((1, "all", N), (2, "uniform", N // 2 + 3), (3, "heavy", 31), (4, "zipf", 0), (5, "zipf", N)):
        new = make(torch, (n, N - n, V, D, "f32", "f32", kind, 0.2), seed, True)
        for k in s:
            s[k].copy_(new[k])
        for k in ("y", "yd", "dE", "dEd"):
            o[k].fill_(MARK)
        g.replay()
        torch.cuda.synchronize()
        check(torch, o, s, n, 1.5, True, "f32")


@pytest.mark.gpu
def test_embed_rows_far_apart():
    """Elements behind the 2^31st of every buffer: the same bits as from rows close together."""
    torch, native = need_gpu()
    N, V, D, ld = 9000, 9000, 40, 245760
    s = make(torch, (N, 0, V, D, "bf16", "bf16", "uniform", 0), 88, False)
    want = run(torch, native, s, 2.0, False)
    far = torch.empty(N, ld, dtype=torch.bfloat16, device="cuda")
    wide = torch.empty(V, ld, dtype=torch.float32, device="cuda")
    apart = {**s, "E": far[:, ld - 48:ld - 8], "dy": far[:, :40]}
    for k in ("E", "dy"):
        apart[k].copy_(s[k])
    o = {"y": far[:, 64:104], "dE": wide[:, ld - 40:], "work": want["work"].clone()}
    run(torch, native, apart, 2.0, False, out=o)
    torch.cuda.synchronize()
    for k in ("y", "dE"):
        assert torch.equal(o[k], want[k]), k


@pytest.mark.gpu
def test_embed_gradient_against_differences():
    """The lookup is linear: <dy, y(E + e D) - y(E)> / e is <dE, D>, and the tangent is y(D)."""
    torch, native = need_gpu()
    s = make(torch, (700, 0, 90, 24, "f32", "f32", "zipf", 0.1), 89, True)
    o = run(torch, native, s, 1.7, True)
    moved = {**s, "E": strided(torch, s["E"] + s["Ed"])}
    m = run(torch, native, moved, 1.7, True)
    torch.cuda.synchronize()
    # three float32 roundings of values below 2^4 each
    assert (m["y"].double() - o["y"].double() - o["yd"].double()).abs().max() <= 3 * 2.0 ** -20
    left = (s["dy"].double() * o["yd"].double()).sum()
    right = (o["dE"].double() * s["Ed"].double()).sum()
    size = (s["dy"].double().abs() * o["yd"].double().abs()).sum()
    assert (left - right).abs() <= size * 1100 * U
