"""lora_kv_attention where a row's scores rise along its tokens: the value that weights are taken against has to move, in small steps, in
large ones, and from scores of ordinary size to ones of thousands, after weights have been summed.

Scores are made of two terms that are exact in fp32, so that what the results are held to is the softmax and not the sums of the scores:
q has a power of two in elements 0 and 1, K a whole number of at most 8 bits in either."""
import math

import pytest
import torch

from kv_common import KvCase, attend, attention64, check_attention

pytestmark = pytest.mark.gpu
LOG2E = math.log2(math.e)


def rising(rows, n, heads, kv, dim, coarse, seed=0, unit=1.0, fine=2.0 ** -4):
    """One sequence.  Score of token j: unit * (coarse(j) + fine * (a number from -128 to 127))."""
    case = KvCase([rows], [n], heads, kv, dim, page=16, seed=seed)
    case.q.zero_()
    case.q.view(rows, heads, dim)[:, :, 0] = unit
    case.q.view(rows, heads, dim)[:, :, 1] = unit * fine
    g = torch.Generator().manual_seed(seed)
    low = torch.randint(-128, 128, (n,), generator=g)
    for j in range(n):
        place = (0, case.table[0, j // 16], slice(None), j % 16)
        case.k5[place] = 0.0
        whole = float(coarse(j))
        assert whole == int(whole) and abs(whole) < 256
        case.k5[place + (0,)] = whole
        case.k5[place + (1,)] = float(low[j])
    return case.device()


def check(case, causal=True, window=0):
    got = attend(case, 1.0, causal, window)
    want = attention64(case, 1.0, causal, window)
    # weights that were summed against a rounded reference of up to 2^12 or 2^13 are off by half a step of it, 2^-12 in
    # powers of two, wherever exact differences take over: 2^-12 more of the weighted |v|
    ref, lse, mag, big = want
    out = got[0].double().cpu()
    bound = mag * (1.02 * 2.0 ** -7 + 2.0 ** -12) + 1e-37
    err = (out - ref).abs()
    assert torch.isfinite(out).all()
    assert (err <= bound).all(), f"worst {float((err / bound).max()):.2f}"
    tol = 2.0 ** -24 * case.dim * big + 2.0 ** -20 * (1 + lse.abs()) + 2.0 ** -12
    e = got[1].double().cpu()
    empty = torch.isinf(lse)
    assert torch.equal(torch.isinf(e) & (e < 0), empty)
    assert ((e - lse).abs() <= tol)[~empty].all()
    assert int(case.batch.status.item()) == 0


SHAPES = [(1, 4, 2, 128), (6, 4, 1, 64), (100, 4, 2, 128), (100, 4, 2, 64), (40, 8, 1, 80), (70, 4, 2, 256), (50, 3, 1, 200)]


@pytest.mark.parametrize("rows,heads,kv,dim", SHAPES)
@pytest.mark.parametrize("per", [1, 7, 64, 100])
def test_scores_that_rise_a_little(rows, heads, kv, dim, per):
    """By one e for every `per` tokens: weights pass any bound again and again."""
    n = 700
    check(rising(rows, n, heads, kv, dim, lambda j: min(250, j // per), seed=per))


@pytest.mark.parametrize("rows,heads,kv,dim", SHAPES)
@pytest.mark.parametrize("at", [63, 64, 200, 460])
@pytest.mark.parametrize("low,high", [(0, 9), (-250, 250), (-100, -93), (-250, -20)])
def test_scores_that_jump_once(rows, heads, kv, dim, at, low, high):
    check(rising(rows, 500, heads, kv, dim, lambda j: high if j >= at else low, seed=at))


@pytest.mark.parametrize("rows,heads,kv,dim", SHAPES)
@pytest.mark.parametrize("unit", [8.0, 32.0, 1024.0])
def test_scores_that_grow_to_thousands(rows, heads, kv, dim, unit):
    """Through the size from which differences are taken before they are scaled (2^12 in powers of two), upwards and, from
    far below zero, towards zero; the fine part is of a few units, so that several tokens count."""
    fine = (2.0 ** -8 if unit < 100 else 2.0 ** -5) / unit       # 24 bits hold the largest score and this
    check(rising(rows, 600, heads, kv, dim, lambda j: j // 3, unit=unit, fine=fine))
    check(rising(rows, 600, heads, kv, dim, lambda j: -255 + j // 3, unit=unit, fine=fine))
    # a plateau on either side of the bound
    edge = int(4096 / LOG2E / unit)
    if 1 <= edge < 250:
        check(rising(rows, 600, heads, kv, dim, lambda j: edge + (j // 128) - 1, unit=unit, fine=fine))


@pytest.mark.parametrize("rows,heads,kv,dim", [(100, 4, 2, 128), (6, 4, 2, 128)])
def test_scores_that_fall(rows, heads, kv, dim):
    check(rising(rows, 700, heads, kv, dim, lambda j: 250 - j // 3))
    check(rising(rows, 700, heads, kv, dim, lambda j: 250 - j // 3), window=90)


def test_rising_in_one_row_of_many():
    """Only some rows' scores rise: the others of the tile must keep what they have."""
    case = rising(120, 640, 4, 2, 128, lambda j: j // 3)
    scale = torch.tensor([2.0 ** -4, 0.0, -1.0, 1.0, 16.0, -64.0]).repeat(20)
    case.q = (case.q.float().view(120, 4, 128) * scale[:, None, None]).view(120, -1).to(torch.bfloat16)
    case.qd = case.q.cuda()
    check(case)
    check(case, window=100)
    check_attention(case, attend(case, 2.0 ** -6, False), attention64(case, 2.0 ** -6, False))
