"""Rows that attend to one key, themselves: softmax over one score is 1 whatever the score, so that
dS and its tangent are zero, not small.  The first row of every sequence is such a row; in
sequences of one token dk, dk' are zero with it."""
import pytest

import attn_ops_util as au
from gpu_util import need_gpu

LENS = {
    "one_token": [1] * 300,
    "mixed": [1, 1, 5, 1, 40, 130, 1, 1, 128, 3, 1],
    # a tile's first row and its last one begin a sequence; one goes on over two tiles
    "tile_edges": [127, 1, 128, 1, 127, 300, 1],
}


@pytest.mark.gpu
@pytest.mark.parametrize("D,dual", [(64, False), (64, True), (40, True), (128, False), (72, False)])
@pytest.mark.parametrize("name", list(LENS))
def test_one_key_has_no_gradient(name, D, dual):
    torch, native = need_gpu()
    lens, Hq, Hkv, tail = LENS[name], 4, 2, 3
    v = au.data(lens, tail, Hq, Hkv, D, dual, seed=21)
    ref, bound = au.reference(v, lens, Hq, Hkv, D)
    out = au.run(native, au.wide(v), lens, Hq, Hkv, D)
    torch.cuda.synchronize()
    au.check(out, ref, bound, sum(lens), dual)
    first = au.starts_of(lens)[:-1].long().cuda()
    alone = first[torch.tensor(lens).cuda() == 1]
    for k in ("dq", "dqd")[:1 + dual]:
        assert not ref[k][first.cpu()].abs().max() > 1e-12
        assert (out[k][first] == 0).all(), (k, out[k][first].abs().max().item())
    for k in ("dk", "dkd")[:1 + dual]:
        assert (out[k][alone] == 0).all(), (k, out[k][alone].abs().max().item())


@pytest.mark.gpu
@pytest.mark.parametrize("D,dual", [(64, True), (128, False)])
def test_one_key_not_finite(D, dual):
    """A NaN in a lone row's value shows in its o and nowhere else."""
    torch, native = need_gpu()
    lens, Hq, Hkv = [1, 1, 1, 50], 2, 1
    v = au.data(lens, 0, Hq, Hkv, D, dual, seed=22)
    want = {k: t.clone() for k, t in au.run(native, au.wide(v), lens, Hq, Hkv, D).items()}
    v["v"][1] = float("nan")
    out = au.run(native, au.wide(v), lens, Hq, Hkv, D)
    torch.cuda.synchronize()
    rest = torch.tensor([0] + list(range(2, 53))).cuda()
    assert torch.isnan(out["o"][1]).all()
    for k in ("o", "dq", "dk", "dv"):
        assert torch.equal(out[k][rest], want[k][rest]), k
