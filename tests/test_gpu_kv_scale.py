"""Attention with scales at the ends of fp32's range."""
import pytest
import torch

from kv_common import KvCase, attend

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("scale", [3.0e38, 2.4e38, 2.3e38, 1.0e30])
@pytest.mark.parametrize("rows", [1, 5, 100])
def test_the_largest_scales_pick_the_largest_score(scale, rows):
    """Scores of 0, 1 and 2 before the scale: the tokens with the largest share the weight, whatever the scale."""
    n = 300
    case = KvCase([rows], [n], 2, 1, 64, seed=rows)
    case.q.zero_()
    case.q.view(rows, 2, 64)[:, :, 0] = 1.0
    for j in range(n):
        place = (0, case.table[0, j // 16], 0, j % 16)
        case.k5[place] = 0.0
        case.k5[place + (0,)] = float(j % 3)
    case.device()
    out, _ = attend(case, scale, lse=False)
    v = case.tokens(0)[1][0]
    for i in range(rows):
        seen = n - rows + i + 1
        want = v[:seen][2::3].mean(0)
        mag = v[:seen][2::3].abs().mean(0)
        err = (out[i].double().cpu().view(2, 64) - want).abs()
        assert (err <= mag * 1.02 * 2.0 ** -7 + 1e-37).all(), i


@pytest.mark.parametrize("scale", [1.5e-45, 1.0e-40, 1.2e-38])
@pytest.mark.parametrize("rows", [1, 100])
def test_the_smallest_scales_weigh_all_tokens_alike(scale, rows):
    case = KvCase([rows], [300], 2, 1, 64, seed=rows).device()
    out, _ = attend(case, scale, lse=False)
    v = case.tokens(0)[1][0]
    for i in range(rows):
        seen = 300 - rows + i + 1
        err = (out[i].double().cpu().view(2, 64) - v[:seen].mean(0)).abs()
        assert (err <= v[:seen].abs().mean(0) * 1.02 * 2.0 ** -7 + 1e-37).all(), i
