"""lora_kv_attention against the definition in 64 bits: head layouts, page sizes, lengths from none to a few
thousand, masks, what pages hold past a sequence, cuts of long ranges, streams and graphs."""
import math

import numpy as np
import pytest
import torch

import paper_2604_07173_amd as L
from kv_common import KvCase, attend, attention64, check_attention

pytestmark = pytest.mark.gpu


def run(case, causal=True, window=0, scale=None, **kw):
    scale = scale or 1.0 / math.sqrt(case.dim)
    case.device()
    got = attend(case, scale, causal, window, **kw)
    torch.cuda.synchronize()
    check_attention(case, got, attention64(case, scale, causal, window, kw.get("layer", 0)))
    return got


@pytest.mark.parametrize("heads,kv,dim", [(8, 2, 128), (4, 4, 64), (8, 1, 128), (6, 2, 80), (4, 4, 8), (7, 7, 40), (12, 2, 96),
                                          (4, 2, 256), (64, 1, 64), (9, 3, 72), (5, 1, 200), (48, 1, 128)])
@pytest.mark.parametrize("slot_major", [False, True])
def test_head_layouts(heads, kv, dim, slot_major):
    run(KvCase([1, 1, 3, 0, 9, 1], [1, 70, 45, 20, 33, 300], heads, kv, dim, slot_major=slot_major, seed=heads + dim))
    run(KvCase([40, 5, 70], [40, 200, 131], heads, kv, dim, slot_major=slot_major, seed=heads + dim + 1))


@pytest.mark.parametrize("page", [1, 2, 4, 8, 16, 32, 64, 128, 1024])
def test_page_sizes(page):
    run(KvCase([1, 2, 1, 1, 50], [1, 31, 32, 33, 97], page=page, seed=page))
    run(KvCase([1, 1], [1023, 1025], page=page, seed=page + 1))


@pytest.mark.parametrize("n", [0, 1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 256, 257, 383, 384, 385, 511, 512,
                               513, 640, 1000, 1537])
def test_lengths_of_one_row(n):
    run(KvCase([1], [n], 8, 2, 128, seed=n))


@pytest.mark.parametrize("rows", [1, 2, 3, 4, 5, 8, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 200, 256, 257])
@pytest.mark.parametrize("ctx", [0, 1, 77])
def test_rows(rows, ctx):
    run(KvCase([rows], [rows + ctx], 8, 2, 128, seed=rows))


@pytest.mark.parametrize("window", [1, 2, 16, 31, 32, 33, 100, 1000, 2**31 - 1])
def test_windows(window):
    run(KvCase([1, 4, 60, 1], [500, 90, 150, 3], seed=window & 255), window=window)
    run(KvCase([150], [300], 4, 2, 128, seed=window & 255), window=window)


@pytest.mark.parametrize("dim", [64, 128, 256])
def test_not_causal(dim):
    run(KvCase([5, 1, 40, 0, 130], [0, 1, 90, 10, 300], dim=dim, seed=5), causal=False)


def test_more_rows_than_tokens():
    """Rows at negative positions see nothing: zeros and -inf."""
    case = KvCase([5, 3, 140], [2, 0, 70], seed=3)
    out, lse = run(case)
    assert not out[:3].any() and torch.isinf(lse[:3]).all() and lse[3:5].isfinite().all()


def test_all_sequences_empty():
    out, lse = run(KvCase([2, 3], [0, 0], seed=1), causal=False)
    assert not out.any() and torch.isinf(lse).all()


def test_no_rows():
    case = KvCase([0, 0], [5, 9], seed=1).device()
    L.lora_kv_attention(case.cache, 0, case.batch, None, 0, 4, None, 0, None, 1.0, torch.empty(256, device="cuda"))


@pytest.mark.parametrize("stale", [float("nan"), float("inf"), -float("inf"), 3.0e38])
def test_stale_slots_have_no_effect(stale):
    run(KvCase([1, 7, 130], [50, 61, 133], 4, 2, 128, page=64, stale=stale, seed=9))


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("rows,window", [(6, 0), (6, 9), (150, 0), (150, 40)])
def test_hidden_tokens_may_hold_anything(bad, rows, window):
    """A token that is no number must not reach rows that cannot see it, though other rows of their tile do."""
    case = KvCase([rows], [rows + 40], 4, 2, 128, seed=2)
    where = 40 + rows // 2
    page, slot = case.table[0, where // 16], where % 16
    case.k5[0, page, :, slot] = bad
    case.v5[0, page, :, slot] = bad
    hidden = [t for t in range(rows) if not (40 + t >= where and (window == 0 or 40 + t < where + window))]
    case.device()
    scale = 1 / math.sqrt(128)
    out, lse = attend(case, scale, True, window)
    clean = KvCase([rows], [rows + 40], 4, 2, 128, seed=2).device()
    want, want_lse = attend(clean, scale, True, window)
    assert torch.equal(out[hidden], want[hidden]) and torch.equal(lse[hidden], want_lse[hidden])
    seen = [t for t in range(rows) if t not in hidden]
    assert torch.isnan(out[seen].float()).all()


def test_large_scores():
    """Scores of thousands: the softmax is one token, or a few that are near."""
    run(KvCase([1, 5, 40, 140], [300, 50, 80, 200], 4, 2, 128, q_scale=300.0, seed=4))


def test_lowest_scores():
    """Keys that all give about the lowest value of the type: equal weights, no overflow."""
    case = KvCase([1, 40], [20, 60], 2, 1, 64, seed=4)
    case.q.fill_(2.0 ** 60)
    case.k5[:] = torch.where(torch.isnan(case.k5), case.k5, torch.full((), -2.0 ** 60, dtype=torch.bfloat16))
    case.device()
    out, lse = attend(case, 2.0 ** -3)
    ref = torch.stack([case.tokens(0)[1][0, :20].mean(0)] + [case.tokens(1)[1][0, :21 + i].mean(0) for i in range(40)])
    got = out.double().cpu().view(41, 2, 64)
    assert torch.isfinite(got).all()
    for h in range(2):
        assert (got[:, h] - ref).abs().max() <= 2.0 ** -7 * 1.02 * 4.5


@pytest.mark.parametrize("lens", [[3000], [5000, 100, 1], [2049, 4097, 513, 8]])
@pytest.mark.parametrize("heads,kv,dim", [(8, 2, 128), (3, 1, 64), (4, 2, 256)])
def test_long_ranges_are_cut_and_joined(lens, heads, kv, dim):
    run(KvCase([1] * len(lens), lens, heads, kv, dim, seed=len(lens)))


@pytest.mark.parametrize("rows,lens", [([9, 2], [2500, 3000]), ([30, 1, 200], [1500, 2000, 900])])
def test_long_ranges_of_several_rows(rows, lens):
    run(KvCase(rows, lens, 4, 1, 128, seed=7))
    run(KvCase(rows, lens, 4, 1, 128, seed=8), window=700)
    run(KvCase(rows, lens, 4, 1, 128, seed=9), causal=False)


def test_many_sequences():
    rng = np.random.default_rng(5)
    lens = rng.integers(0, 60, 700).tolist()
    rows = [int(min(n, r)) for n, r in zip(lens, rng.integers(0, 3, 700))]
    run(KvCase(rows, lens, 2, 1, 64, seed=6))


def test_more_sequences_than_a_wave_finds_at_once():
    lens = [1 + i % 3 for i in range(5000)]
    run(KvCase([1] * 5000, lens, 1, 1, 8, page=4, seed=6))


def test_unknown_or_wrong_longest_chunk():
    """max_rows decides which kernels run, never what comes out."""
    for given in (0, 1, 7, 1000):
        run(KvCase([3, 0, 50, 1, 133], [30, 20, 77, 5, 140], 4, 2, 128, seed=11, max_rows=given))
    # as if all sequences had as many
    run(KvCase([1, 0, 9, 2, 3], [30, 20, 77, 5, 140], 4, 2, 128, seed=11, max_rows=3))
    run(KvCase([40, 0, 50, 10, 0], [40, 20, 77, 15, 140], 4, 2, 128, seed=11, max_rows=20))


def test_strides_and_layers():
    case = KvCase([2, 40], [40, 60], 4, 2, 64, layers=3, wide=72, seed=12).device()
    for layer in (2, 0):
        out, lse = attend(case, 0.125, layer=layer, ldo=4 * 64 + 24)
        check_attention(case, (out, lse), attention64(case, 0.125, layer=layer))
        assert (out[:, 256:] == 7.0).all()


def test_bit_identical_run_to_run():
    case = KvCase([1, 9, 140], [3000, 50, 700], 8, 2, 128, seed=13).device()
    a = attend(case, 0.1)
    for _ in range(3):
        b = attend(case, 0.1)
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_without_lse():
    case = KvCase([1, 40], [600, 50], 8, 2, 128, seed=13).device()
    a, b = attend(case, 0.1), attend(case, 0.1, lse=False)
    assert torch.equal(a[0], b[0])


def test_a_page_outside_the_cache_raises_the_status_bit():
    case = KvCase([1, 1, 40], [40, 40, 60], seed=14)
    good = attention64(case, 0.125)
    case.table[1, 1] = 10 ** 6
    case.device()
    out, lse = attend(case, 0.125)
    assert int(case.batch.status.item()) == L.LORA_STATUS_BAD_PAGE
    case.batch.status.zero_()
    keep = [0] + list(range(2, 42))
    sub = lambda t: t[keep]                                                       # noqa: E731
    assert ((out.double().cpu()[keep] - sub(good[0])).abs() <= sub(good[2]) * 1.02 * 2.0 ** -7).all()


def test_a_length_beyond_the_table_raises_the_status_bit():
    case = KvCase([1, 1], [40, 48], seed=15).device()
    case.batch.seq_len[1] = 10 ** 9
    attend(case, 0.125)
    assert int(case.batch.status.item()) == L.LORA_STATUS_BAD_LENGTH
    case.batch.status.zero_()
    case.batch.seq_len[1] = -5
    attend(case, 0.125)
    assert int(case.batch.status.item()) == L.LORA_STATUS_BAD_LENGTH


@pytest.mark.parametrize("n", [4, 300])
@pytest.mark.parametrize("place,value", [(0, 1), (2, 1), (2, -3), (3, 10 ** 6), (-1, 5)])
def test_rows_that_are_no_partition_raise_the_status_bit_and_write_nothing(n, place, value):
    case = KvCase([2] * (n - 1) + [70], [40] * (n - 1) + [90], seed=17).device()
    case.batch.row_start[place] = value
    out, lse = attend(case, 0.125)                                                # which fills both with 7 before
    assert int(case.batch.status.item()) == L.LORA_STATUS_BAD_LENGTH
    assert (out == 7.0).all() and (lse == 7.0).all()


def test_another_stream():
    case = KvCase([1, 60], [700, 90], 8, 2, 128, seed=16).device()
    torch.cuda.synchronize()
    want = attend(case, 0.1)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        got = attend(case, 0.1)
    s.synchronize()
    assert torch.equal(want[0], got[0]) and torch.equal(want[1], got[1])
    out, ws = torch.zeros_like(want[0]), torch.empty(L.lora_kv_attention_ws_bytes(case.cache, case.batch, 8), dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    L.lora_kv_attention(case.cache, 0, case.batch, case.qd, 1024, 8, out, 1024, None, 0.1, ws, stream=s)
    s.synchronize()
    assert torch.equal(want[0], out)


def test_in_a_graph():
    case = KvCase([1, 1, 70], [900, 40, 90], 8, 2, 128, seed=17).device()
    scale = 0.09
    ws = torch.empty(L.lora_kv_attention_ws_bytes(case.cache, case.batch, 8), dtype=torch.uint8, device="cuda")
    out = torch.zeros((case.T, 8 * 128), dtype=torch.bfloat16, device="cuda")
    call = lambda: L.lora_kv_attention(case.cache, 0, case.batch, case.qd, 1024, 8, out, 1024, None, scale, ws)   # noqa: E731
    call()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    for i in range(4):
        case.qd.normal_()
        case.batch.seq_len[0] = 900 - 100 * i          # lengths are read on the device
        want, _ = attend(case, scale, lse=False)
        out.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want), i


def test_offsets_beyond_32_bits():
    """Pages whose elements lie past 2^31 in K and V."""
    D, page, kv = 128, 16, 2
    each = kv * page * D
    n_pages = (1 << 31) // each + 40
    k, v = (torch.empty((1, n_pages, kv, page, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    small = KvCase([1, 50], [100, 70], 4, kv, D, seed=18).device()
    far = torch.from_numpy(small.table.astype(np.int64)).cuda() + (n_pages - small.n_pages)
    k[0, n_pages - small.n_pages:] = small.kd[0]
    v[0, n_pages - small.n_pages:] = small.vd[0]
    want = attend(small, 0.1)
    small.cache = L.KvCache(k, v)
    small.batch = L.KvBatch(small.batch.row_start, small.batch.seq_len, far.int().contiguous(), small.T, max_rows=50)
    got = attend(small, 0.1)
    assert torch.equal(want[0], got[0]) and torch.equal(want[1], got[1])
