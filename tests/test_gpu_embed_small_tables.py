"""The gradient of an embedding where a row of the table has thousands of tokens, and where the table is
wide beyond what one launch takes, on both sides of each border (test_embed_rule_cpu.py)."""
import pytest

from gpu_util import need_gpu
from test_gpu_embed import check, make, run

CASES = {
    "one_id_one_launch": (1024, 3, 1, 130, "f32", "bf16", "uniform", 0),
    "one_id_sorted": (1025, 3, 1, 130, "f32", "f32", "uniform", 0),
    "one_id_most": (6144, 0, 1, 24, "f32", "bf16", "uniform", 0),
    "one_id_and_padding": (6000, 0, 1, 7, "f32", "f32", "uniform", 0.4),
    "two_ids": (2049, 0, 2, 300, "f32", "bf16", "heavy", 0.1),
    "five_ids": (6144, 11, 5, 128, "f32", "f32", "zipf", 0.1),
    "six_ids": (6144, 0, 6, 128, "f32", "f32", "zipf", 0),
    "wide_one_launch": (200, 0, 90, 38 * 128, "f32", "bf16", "zipf", 0.1),
    "wide_sorted": (200, 5, 90, 76 * 128 + 1, "f32", "bf16", "zipf", 0.1),
    "wide_sorted_f32": (300, 0, 70, 20001, "f32", "f32", "heavy", 0),
}


@pytest.mark.gpu
@pytest.mark.parametrize("dual", [False, True])
@pytest.mark.parametrize("name", list(CASES))
def test_gradient(name, dual):
    torch, native = need_gpu()
    case = CASES[name]
    s = make(torch, case, 91, dual)
    o = run(torch, native, s, 1.3, dual)
    torch.cuda.synchronize()
    check(torch, o, s, case[0], 1.3, dual, case[5])
