"""lora_kv_share against its definition: whole numbers, so equal."""
import numpy as np
import pytest
import torch

import paper_2604_07173_amd as L
from kv_shared_common import SharedCase, expected_share, random_case, share

pytestmark = pytest.mark.gpu


def check(case, sh, **kw):
    want = expected_share(case.table.tolist(), case.lens, case.rows, case.start.tolist(), case.page, sh.rows.numel(), **kw)
    for name, w in want.items():
        assert getattr(sh, name).tolist() == w, name


@pytest.mark.parametrize("seqs,prompts,most,page,prompt_hi", [
    (1, 1, 1, 16, 60), (2, 1, 1, 16, 60), (3, 1, 2, 1, 20), (17, 2, 1, 8, 400), (64, 4, 1, 16, 900), (63, 9, 5, 4, 300), (65, 30, 1, 2, 40),
    (128, 1, 1, 64, 900), (200, 12, 3, 1, 600), (300, 40, 8, 16, 900), (1024, 100, 2, 8, 300), (1025, 3, 1, 16, 200), (2500, 700, 3, 4, 30)])
def test_groups_are_those_of_the_definition(seqs, prompts, most, page, prompt_hi):
    """One launch and three, arrays in LDS and in memory, one round of a workgroup and several."""
    case = random_case(seqs + prompts, seqs, prompts, most=most, prompt_hi=prompt_hi, own_hi=20, heads=1, kv=1, dim=8, page=page).device()
    check(case, share(case))
    assert int(case.batch.status) == 0


@pytest.mark.parametrize("min_pages", [1, 2, 7, 40])
@pytest.mark.parametrize("max_rows", [0, 1, 3])
def test_what_takes_part(min_pages, max_rows):
    case = random_case(5, 90, 6, most=4, prompt_hi=500, own_hi=200, heads=1, kv=1, dim=8).device()
    check(case, share(case, min_pages, max_rows, room=case.T if not max_rows else min(case.T, 90 * max_rows)), min_pages=min_pages, max_rows=max_rows)


def raw(table, lens, rows, page):
    """A batch over any table."""
    case = SharedCase([-1], [], [0], [1], heads=1, kv=1, dim=8, page=page)
    case.table, case.lens, case.rows = np.array(table, np.int32), list(lens), list(rows)
    case.T, case.start = sum(rows), np.concatenate([[0], np.cumsum(rows)]).astype(np.int32)
    case.max_rows = 0
    return case.device()


@pytest.mark.parametrize("seqs,width", [(40, 12), (300, 12), (60, 700)])
def test_tables_of_any_kind(seqs, width):
    """Few page numbers, so that tables agree and differ anywhere, entries that are no pages among them."""
    rng = np.random.default_rng(seqs + width)
    table = rng.integers(-1, 2, (seqs, width)) * rng.integers(0, 2 ** 31 - 1)
    table[:, 3:] = np.where(rng.random((seqs, 1)) < 0.7, table[:1, 3:], table[:, 3:])
    rows = rng.integers(0, 4, seqs)
    lens = np.minimum(rng.integers(0, width * 4 + 1, seqs) + rows, width * 4)
    for min_pages in (1, 3, 9, width, width + 1):
        case = raw(table, lens.tolist(), rows.tolist(), 4)
        check(case, share(case, min_pages), min_pages=min_pages)


def test_page_numbers_that_meet_in_the_hash_table():
    """All pages multiples of a power of two: their low bits, and many hashes, are the same."""
    n = 500
    table = np.repeat(np.arange(n // 2) << 20, 2)[:, None] + np.zeros((1, 2), int)
    case = raw(table, [8] * n, [1] * n, 4)
    sh = share(case)
    check(case, sh)
    assert sh.counts.tolist() == [n // 2, n, n, n // 2 * 4]
    case = raw(table, [9] * n, [1] * n, 4)           # a token more than the table has room for
    sh = share(case)
    assert sh.counts.tolist() == [0] * 4 and sh.own.tolist() == [0] * n
    assert int(case.batch.status) == L.LORA_STATUS_BAD_LENGTH


def test_a_member_that_is_shorter_limits_the_group():
    case = SharedCase([0, 0, 0], [64], [0, 0, 0], [1, 1, 1], heads=1, kv=1, dim=8)
    case.lens[1] = 40                                # its new row stands inside the third page
    case.device()
    sh = share(case)
    check(case, sh)
    assert sh.groups.tolist() == [[0, 32, 0, 3]] and sh.own.tolist() == [32] * 3


@pytest.mark.parametrize("lens,start", [([-1, 50, 50, 50], None), ([50, 5000, 50, 50], None), ([50] * 4, [0, 2, 1, 3, 4]), ([50] * 4, [0, 1, 2, 3, 9]),
                                        ([50] * 4, [1, 1, 2, 3, 4]), ([50] * 4, [0, 1, 2, 3, 3])])
def test_lengths_and_rows_that_make_no_sense(lens, start):
    case = SharedCase([0] * 4, [48], [1] * 4, [1] * 4, heads=1, kv=1, dim=8)
    case.lens = lens
    if start:
        case.start = np.array(start, np.int32)
    case.device()
    sh = share(case)
    assert int(case.batch.status) == L.LORA_STATUS_BAD_LENGTH
    if start:                                        # no partition: no groups
        assert sh.counts.tolist() == [0] * 4 and sh.own.tolist() == [0] * 4 and sh.place.tolist() == [-1] * 4
        assert sh.groups.tolist() == [[-1, 0, 0, 0]] * 2 and sh.rows.tolist() == [-1] * 4
    else:
        bad = 0 if lens[0] < 0 else 1
        own = [48 if s != bad else 0 for s in range(4)]
        assert sh.own.tolist() == own and sh.counts.tolist() == [1, 3, 3, 96]


def test_another_stream_and_repeated_calls_in_a_graph():
    case = random_case(3, 80, 5, most=2, prompt_hi=200, heads=1, kv=1, dim=8).device()
    want = share(case)
    sh = share(case)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        L.lora_kv_share(case.cache, case.batch, sh)
    for fill in (0, -5, 1 << 30):
        for t in (sh.groups, sh.rows, sh.own, sh.place, sh.counts):
            t.fill_(fill)
        sh.ws.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        for name in ("groups", "rows", "own", "place", "counts"):
            assert torch.equal(getattr(sh, name), getattr(want, name))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = share(case, stream=side)
    side.synchronize()
    # the fills of share() ran on the other stream: run again behind them
    torch.cuda.synchronize()
    L.lora_kv_share(case.cache, case.batch, got, stream=side)
    side.synchronize()
    assert torch.equal(got.groups, want.groups) and torch.equal(got.rows, want.rows)


def test_a_batch_without_rows_leaves_the_results_of_the_call_before():
    case = random_case(3, 20, 2, most=1, prompt_hi=200, heads=1, kv=1, dim=8).device()
    want, sh = share(case), share(case)
    none = L.KvBatch(torch.zeros_like(case.batch.row_start), case.batch.seq_len, case.batch.table, n_rows=0)
    L.lora_kv_share(case.cache, none, sh)
    torch.cuda.synchronize()
    assert int(sh.counts[0]) > 0 and int(none.status) == 0
    for name in ("groups", "rows", "own", "place", "counts"):
        assert torch.equal(getattr(sh, name), getattr(want, name))
