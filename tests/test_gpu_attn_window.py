"""Windowed packed attention with sinks (mf_attn_window_fwd / mf_attn_window_bwd) against the float64
definition, element by element within bounds derived from the roundings: windows of one row and
around every tile edge, sinks in a sequence's own tile, across tiles and across the chunks of query
rows that sum their gradients, sequences shorter than their sinks, grouped heads, tangents, rows
behind the last sequence, values that are not finite where nothing attends, streams, graphs."""
import math

import pytest

import attn_ops_util as au
import attn_window_util as wu
from gpu_util import need_gpu

CASES = {
    # lens, tail, Hq, Hkv, D, window, sinks
    "one_token": ([1, 1], 0, 1, 1, 64, 1, 1),
    "itself": ([130, 1, 60], 3, 2, 1, 64, 1, 0),
    "itself_and_sinks": ([130, 1, 60], 3, 2, 1, 64, 1, 5),
    "two": ([70, 129], 0, 4, 2, 16, 2, 0),
    "below_tile": ([300, 100], 5, 2, 2, 64, 63, 0),
    "tile": ([300, 100], 0, 2, 1, 64, 64, 4),
    "above_tile": ([300, 100], 0, 2, 1, 40, 65, 4),
    "rows": ([390], 0, 4, 2, 64, 128, 1),
    "above_rows": ([390, 7], 1, 2, 1, 64, 129, 64),
    "many_short": ([3, 5, 1, 7, 2, 9, 0, 4, 8, 6, 1, 1, 30, 17, 2, 90, 12], 2, 2, 2, 16, 4, 2),
    "many_sequences": ([0, 1, 2, 0, 1, 3] * 380, 1, 2, 1, 16, 2, 1),
    # sinks whose sequence goes on over the chunks of 512 query rows
    "chunks": ([1300], 0, 2, 1, 64, 50, 4),
    "chunks_all_sinks": ([500, 30, 1100], 9, 2, 2, 64, 100, 128),
    "sinks_across_tiles": ([510, 700], 0, 2, 1, 24, 5, 17),
    "sinks_at_border": ([512, 700], 0, 4, 2, 64, 33, 8),
    "short_over_border": ([511, 60, 700], 0, 2, 1, 64, 1, 128),
    "window_over_border": ([400, 500, 300], 3, 2, 1, 64, 300, 3),
    "chunk_group": ([100, 1000], 0, 8, 1, 32, 90, 16),
    "chunk_group_10": ([600, 50], 0, 10, 1, 24, 30, 3),
    # chunks of 1024
    "long": ([2300], 0, 2, 1, 64, 600, 3),
    "long_two": ([900, 1500], 7, 1, 1, 64, 513, 100),
}
WIDE = {
    "wide_edges": ([128, 1, 0, 255, 64], 7, 4, 2, 128, 70, 2),
    "wide_72": ([130, 66], 1, 2, 2, 72, 128, 0),
    "wide_chunks": ([40, 1150], 0, 3, 1, 128, 127, 9),
    "wide_96_grouped": ([700], 0, 8, 1, 96, 200, 128),
}
RUNS = [(n, d) for n in CASES for d in (False, True)] + [(n, False) for n in WIDE]


def _reference(v, *a, **kw):
    return wu.reference({k: t.cuda() for k, t in v.items()}, *a, **kw)


@pytest.mark.gpu
@pytest.mark.parametrize("name,dual", RUNS)
def test_window_against_definition(name, dual):
    torch, native = need_gpu()
    lens, tail, Hq, Hkv, D, window, sinks = {**CASES, **WIDE}[name]
    v = au.data(lens, tail, Hq, Hkv, D, dual, seed=61)
    ref, bound = _reference(v, lens, Hq, Hkv, D, window, sinks)
    out = wu.run(native, au.wide(v), lens, Hq, Hkv, D, window, sinks)
    torch.cuda.synchronize()
    au.check(out, ref, bound, sum(lens), dual)


@pytest.mark.gpu
@pytest.mark.parametrize("D,dual", [(64, False), (64, True), (128, False)])
def test_window_large_scores_and_scale(D, dual):
    """Scores of several hundred: rows that are one key, a sink or one in the window."""
    torch, native = need_gpu()
    lens, Hq, Hkv = [150, 700], 2, 1
    v = au.data(lens, 0, Hq, Hkv, D, dual, seed=62, qstd=12.0)
    ref, bound = _reference(v, lens, Hq, Hkv, D, 90, 6, scale=0.75)
    out = wu.run(native, au.wide(v), lens, Hq, Hkv, D, 90, 6, scale=0.75)
    torch.cuda.synchronize()
    au.check(out, ref, bound, sum(lens), dual)


@pytest.mark.gpu
@pytest.mark.parametrize("D,dual", [(64, False), (64, True), (128, False)])
def test_window_of_all_rows_is_attention(D, dual):
    """A window that holds every row: the bits of the calls without one; one that holds every row of a
    sequence but not of the batch: within the bounds of those."""
    torch, native = need_gpu()
    lens, tail, Hq, Hkv = [300, 1, 77], 5, 4, 2
    v = au.data(lens, tail, Hq, Hkv, D, dual, seed=63)
    w = au.wide(v)
    want = au.run(native, w, lens, Hq, Hkv, D)
    for window, sinks in ((383, 0), (2 ** 31 + 7, 128), (2 ** 62, 3)):
        got = wu.run(native, w, lens, Hq, Hkv, D, window, sinks)
        for k in au.names(dual):
            assert torch.equal(got[k], want[k]), (window, k)
    ref, bound = au.reference(v, lens, Hq, Hkv, D)
    for window, sinks in ((382, 0), (300, 7)):
        got = wu.run(native, w, lens, Hq, Hkv, D, window, sinks)
        torch.cuda.synchronize()
        au.check(got, ref, bound, sum(lens), dual)


@pytest.mark.gpu
@pytest.mark.parametrize("n,length", [(1, 700), (300, 1), (5, 60), (2, 600)])
@pytest.mark.parametrize("D,dual", [(64, True), (128, False)])
def test_window_equal_sequences_by_their_number(D, dual, n, length):
    torch, native = need_gpu()
    v = au.wide(au.data([length] * n, 0, 4, 2, D, dual, seed=64))
    want = wu.run(native, v, [length] * n, 4, 2, D, 40, 3)
    got = wu.run(native, v, None, 4, 2, D, 40, 3, n_seq=n)
    torch.cuda.synchronize()
    assert int(got["status"].item()) == 0
    for k in au.names(dual):
        assert torch.equal(got[k], want[k]), k


@pytest.mark.gpu
@pytest.mark.parametrize("D,dual", [(64, False), (64, True), (128, False), (40, True)])
@pytest.mark.parametrize("poison", [math.nan, math.inf, -math.inf])
def test_window_masked_places_do_not_matter(D, dual, poison):
    """What a row does not attend to never reaches it: rows that its window has left behind, rows
    behind the last sequence, all of another sequence."""
    torch, native = need_gpu()
    lens, tail, Hq, Hkv, window, sinks = [300, 45, 900, 20], 33, 2, 1, 50, 3
    n = sum(lens)
    clean = au.data(lens, tail, Hq, Hkv, D, dual, seed=65)
    want = {k: t.clone() for k, t in wu.run(native, au.wide(clean), lens, Hq, Hkv, D, window, sinks).items()}
    # a row of the first sequence, the whole second one, a row far behind the third's sinks, the rest
    bad = [100] + list(range(300, 345)) + [945] + list(range(n, n + tail))
    dirty = {k: t.clone() for k, t in clean.items()}
    for t in dirty.values():
        t[bad] = poison
    got = wu.run(native, au.wide(dirty), lens, Hq, Hkv, D, window, sinks)
    torch.cuda.synchronize()
    assert int(got["status"].item()) == 0
    # rows that attend to a poisoned one, and keys that such a row attends to
    hit = set(range(100, 150)) | set(range(300, 345)) | set(range(945, 995))
    keys = hit | set(range(51, 100)) | set(range(896, 945)) | {0, 1, 2, 345, 346, 347}
    rows = torch.tensor([r for r in range(n) if r not in hit]).cuda()
    kept = torch.tensor([r for r in range(n) if r not in keys]).cuda()
    for k in au.names(dual):
        a, b = (got[k].t(), want[k].t()) if k in ("lse", "rbar") else (got[k], want[k])
        at = kept if k in ("dk", "dv", "dkd", "dvd") else rows
        assert torch.equal(a[at], b[at]), k
        assert (a[n:] == au.MARK).all(), k
    for k in au.names(dual, False):
        a = got[k].t() if k in ("lse", "rbar") else got[k]
        assert not torch.isfinite(a[sorted(hit)]).all(1).any(), k
    for k in ("dk", "dv"):
        assert not torch.isfinite(got[k][sorted(keys)]).all(1).any(), k


@pytest.mark.gpu
@pytest.mark.parametrize("which", ["qd", "kd", "vd", "dod"])
def test_window_tangents_stay_among_themselves(which):
    """Tangents that are not finite reach tangents alone."""
    torch, native = need_gpu()
    lens, Hq, Hkv, D, window, sinks = [70, 645], 4, 2, 64, 30, 2
    v = au.data(lens, 3, Hq, Hkv, D, True, seed=66)
    want = {k: t.clone() for k, t in wu.run(native, au.wide(v), lens, Hq, Hkv, D, window, sinks).items()}
    v[which][[3, 71, 400, 717]] = math.nan
    out = wu.run(native, au.wide(v), lens, Hq, Hkv, D, window, sinks)
    torch.cuda.synchronize()
    for k in ("o", "lse", "dq", "dk", "dv"):
        assert torch.equal(out[k], want[k]), k
    seen = {"qd": "od", "kd": "od", "vd": "od", "dod": "dvd"}[which]
    assert not torch.isfinite(out[seen][[3, 71, 400]]).all(1).any()
    clear = list(range(3)) + list(range(33, 71))
    if which != "dod":
        assert torch.equal(out["od"][clear], want["od"][clear])


@pytest.mark.gpu
@pytest.mark.parametrize("D,dual", [(64, True), (128, False)])
def test_window_sequences_do_not_feel_one_another(D, dual):
    """A sequence's bits do not depend on what shares its tiles and chunks."""
    torch, native = need_gpu()
    lens, Hq, Hkv = [40, 77, 700, 3, 130, 60], 4, 2
    v = au.data(lens, 9, Hq, Hkv, D, dual, seed=67)
    run = lambda w: wu.run(native, au.wide(w), lens, Hq, Hkv, D, 45, 5)
    want = {k: t.clone() for k, t in run(v).items()}
    mine = [r for r in range(sum(lens)) if 117 <= r < 817 or 820 <= r < 950]
    others = [r for r in range(sum(lens) + 9) if r not in mine]
    for scale in (30.0, 1e18):
        w = {k: t.clone() for k, t in v.items()}
        for t in w.values():
            t[others] = (t[others].float() * scale).bfloat16()
        got = run(w)
        torch.cuda.synchronize()
        for k in au.names(dual):
            a, b = (got[k].t(), want[k].t()) if k in ("lse", "rbar") else (got[k], want[k])
            assert torch.equal(a[mine], b[mine]), (scale, k)


@pytest.mark.gpu
@pytest.mark.parametrize("D,dual", [(64, True), (128, False)])
def test_window_calls_at_once_and_again(D, dual):
    """The same bits again, and from calls that overlap on two streams."""
    torch, native = need_gpu()
    jobs = []
    for seed, lens, window, sinks in ((1, [700, 90], 33, 4), (2, [64, 400, 900], 200, 128)):
        v = au.wide(au.data(lens, 0, 4, 2, D, dual, seed=seed))
        a = (lens, 4, 2, D, window, sinks)
        jobs.append((v, a, {k: t.clone() for k, t in wu.run(native, v, *a).items()}))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in jobs]
    for _ in range(10):
        outs = []
        for (v, a, _), s in zip(jobs, streams):
            with torch.cuda.stream(s):
                outs.append(wu.run(native, v, *a))
        torch.cuda.synchronize()
        for (_, _, want), got in zip(jobs, outs):
            for k in au.names(dual):
                assert torch.equal(got[k], want[k]), k


@pytest.mark.gpu
@pytest.mark.parametrize("D,dual", [(64, True), (128, False)])
def test_window_captured_with_other_lengths(D, dual):
    """A captured call replayed after the lengths on the device have changed (fewer rows too)."""
    torch, native = need_gpu()
    Hq, Hkv, N, window, sinks = 2, 1, 1200, 60, 7
    sets = [[1200], [10, 900, 290], [512, 0, 650], [505, 600]]
    v = au.data([N], 0, Hq, Hkv, D, dual, seed=68)
    w = au.wide(v)
    starts = torch.zeros(4, dtype=torch.int32, device="cuda")

    def put(lens):
        s = au.starts_of(lens)
        starts.copy_(torch.cat([s, s[-1:].expand(4 - len(s))]))

    put(sets[0])
    out = wu.run(native, w, None, Hq, Hkv, D, window, sinks, starts=starts)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        wu.run(native, w, None, Hq, Hkv, D, window, sinks, starts=starts, out=out)
    for lens in sets:
        put(lens)
        for k in au.names(dual):
            out[k].fill_(au.MARK)
        g.replay()
        torch.cuda.synchronize()
        n = sum(lens)
        ref, bound = _reference({k: t[:n] for k, t in v.items()}, lens, Hq, Hkv, D, window, sinks)
        au.check(out, ref, bound, n, dual)


@pytest.mark.gpu
def test_window_sequences_out_of_order_stay_inside():
    """Wrong contents of seq_start give undefined rows, but no access outside the buffers and no
    endless walk: every row index is clamped to the rows."""
    torch, native = need_gpu()
    Hq, Hkv, D, N = 2, 1, 64, 1260
    v = au.wide(au.data([N], 0, Hq, Hkv, D, True, seed=69))
    for s in ([0, 200, 100, 1260], [5, -7, 10 ** 9, 2 ** 31 - 1], [0, 0, 0, -5], [1300, 1300, 1300, 1260],
              [600, 3, 1200, 1000]):
        starts = torch.tensor(s, dtype=torch.int32, device="cuda")
        out = wu.run(native, v, None, Hq, Hkv, D, 20, 100, starts=starts)
        torch.cuda.synchronize()
        assert int(out["status"].item()) == 0


@pytest.mark.gpu
def test_window_no_rows():
    torch, native = need_gpu()
    for N in (0, 40, 1100):
        v = au.wide(au.data([0], N, 2, 1, 64, True, seed=70))
        out = wu.run(native, v, [0], 2, 1, 64, 8, 2)
        torch.cuda.synchronize()
        au.check(out, {}, {}, 0, True)


@pytest.mark.gpu
def test_window_more_row_tiles_than_a_grid_is_high():
    """Tiles behind the 65535th, with the chunks' CTAs among them: the same bits as those rows by
    themselves."""
    torch, native = need_gpu()
    D, n = 8, 65535 * 128 + 512 - 128 + 1024
    n -= n % 1024
    g = torch.Generator(device="cuda").manual_seed(71)
    v = {k: torch.randn(n, D, generator=g, device="cuda").bfloat16() for k in ("q", "k", "v", "do")}
    outs = []
    for rows in (n, 1024):
        w = {k: t[n - rows:] for k, t in v.items()}
        starts = torch.arange(0, rows + 1, 1024, dtype=torch.int32, device="cuda")
        outs.append(wu.run(native, w, None, 1, 1, D, 20, 2, starts=starts))
    torch.cuda.synchronize()
    assert int(outs[0]["status"].item()) == 0
    for k in au.names(False):
        a, b = outs[0][k], outs[1][k]
        a = a[:, n - 1024:] if k == "lse" else a[n - 1024:]
        assert torch.equal(a, b) and torch.isfinite(b).all(), k
        assert not (outs[0][k] == au.MARK).all(), k
