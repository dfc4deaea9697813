"""Attention of sequences that share pages, against the definition in 64 bits (which knows of no sharing)."""
import numpy as np
import pytest
import torch

import paper_2604_07173_amd as L
from kv_common import attend, attention64, check_attention
from kv_shared_common import SharedCase, attend_shared, random_case, share

pytestmark = pytest.mark.gpu


def check(case, sh=None, causal=True, layer=0, scale=None, **kw):
    case.device()
    sh = sh or share(case)
    scale = scale or case.dim ** -0.5
    got = attend_shared(case, sh, scale, causal=causal, layer=layer, **kw)
    check_attention(case, got, attention64(case, scale, causal=causal, layer=layer))
    return got, sh


@pytest.mark.parametrize("heads,kv,dim", [(4, 2, 64), (32, 8, 128), (8, 8, 40), (20, 5, 80), (2, 1, 256), (64, 1, 64), (6, 2, 8), (9, 3, 96)])
@pytest.mark.parametrize("width", [2, 9, 40])
def test_answers_to_one_prompt(heads, kv, dim, width):
    """Groups of few rows and of several tiles."""
    check(SharedCase([0] * width, [203], [i * 7 % 31 for i in range(width)], [1] * width, heads=heads, kv=kv, dim=dim, seed=width))


@pytest.mark.parametrize("page,slot_major", [(1, False), (8, True), (16, False), (64, True), (512, False)])
def test_pages(page, slot_major):
    case = random_case(page, 20, 3, most=3, prompt_hi=1100, own_hi=90, heads=8, kv=2, dim=64, page=page, slot_major=slot_major)
    check(case)


@pytest.mark.parametrize("seqs,prompts,most,prompt_hi,own_hi", [
    (1, 1, 1, 100, 10), (2, 1, 1, 40, 1), (5, 5, 1, 300, 40), (30, 4, 6, 700, 200), (61, 9, 5, 400, 100), (100, 2, 1, 2500, 20), (256, 16, 1, 300, 60),
    (300, 30, 2, 200, 30), (7, 2, 40, 900, 300)])
def test_mixtures_of_groups_and_others(seqs, prompts, most, prompt_hi, own_hi):
    """Sequences in no group, paused ones, prompts without a whole page, plans in LDS and in memory."""
    check(random_case(seqs * 3 + most, seqs, prompts, most=most, prompt_hi=prompt_hi, own_hi=own_hi, heads=8, kv=4, dim=64))


@pytest.mark.parametrize("causal", [True, False])
def test_masks(causal):
    check(random_case(11, 24, 3, most=4, prompt_hi=400, own_hi=50, heads=8, kv=2, dim=64), causal=causal)


@pytest.mark.parametrize("width,tokens", [(3, 9000), (70, 6000)])
def test_a_long_prompt_is_cut(width, tokens):
    """More units of tokens than tiles: parts are joined, of short tiles and of long ones."""
    check(SharedCase([0] * width, [tokens], [5] * width, [1] * width, heads=4, kv=1, dim=64))


@pytest.mark.parametrize("hint", [0, 1, 3, 1000])
def test_hints_of_the_host(hint):
    """The rows of the largest group decide which kernels run; wrong ones too give right results."""
    case = random_case(2, 40, 2, most=3, prompt_hi=500, own_hi=40, heads=8, kv=2, dim=64, max_rows=hint)
    case.device()
    check(case, share(case, max_group_rows=hint))


def test_entries_of_the_others_tables_for_shared_tokens_are_not_looked_at():
    case = SharedCase([0] * 6, [160], [3] * 6, [1] * 6)
    case.device()
    sh = share(case)
    want = attention64(case, 0.125)
    case.batch.table[1:, :10] = -12345
    got = attend_shared(case, sh, 0.125)
    check_attention(case, got, want)


def test_layers_row_strides_and_no_log():
    case = random_case(21, 18, 3, most=2, prompt_hi=300, layers=3, heads=4, kv=2, dim=64)
    case.device()
    sh = share(case)
    for layer in (0, 2):
        out, e = attend_shared(case, sh, 0.2, layer=layer, ldo=4 * 64 + 24)
        check_attention(case, (out, e), attention64(case, 0.2, layer=layer))
        assert (out[:, 256:] == 7.0).all()           # columns behind a row stay
        assert torch.equal(attend_shared(case, sh, 0.2, layer=layer, lse=False)[0], out[:, :256])


def test_bits_repeat_and_batches_without_groups_agree_with_the_plain_call():
    case = random_case(8, 50, 6, most=2, prompt_hi=900, heads=8, kv=2, dim=128).device()
    sh = share(case)
    first = attend_shared(case, sh, 0.09)
    for _ in range(3):
        again = attend_shared(case, sh, 0.09)
        assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])
    alone = share(case, min_pages=1 << 20)           # nobody has as many pages
    assert alone.counts.tolist() == [0] * 4
    want = attention64(case, 0.09)
    check_attention(case, attend_shared(case, alone, 0.09), want)
    check_attention(case, attend(case, 0.09), want)


def test_large_scores_and_infinities_in_shared_tokens():
    case = SharedCase([0] * 5, [96], [0, 4, 20, 1, 9], [1] * 5, heads=4, kv=2, dim=64, q_scale=60.0)
    check(case, scale=3.0)
    page = int(case.table[0, 2])
    case.v5[0, page, 1, 5, 7] = float("inf")
    case.device()
    out = attend_shared(case, share(case), 0.01)[0].view(5, 4, 64)
    bad = ~torch.isfinite(out)
    assert bad[:, 2:, 7].all() and int(bad.sum()) == 5 * 2


def test_rows_that_are_no_partition_write_nothing():
    case = SharedCase([0] * 4, [64], [2] * 4, [1] * 4).device()
    sh = share(case)
    case.batch.row_start[2] = 0
    out, e = attend_shared(case, sh, 0.125)
    assert (out == 7.0).all() and (e == 7.0).all()
    assert int(case.batch.status) == L.LORA_STATUS_BAD_LENGTH


def test_groups_that_are_not_true_stay_within_bounds():
    """Numbers out of every range: rows of no group are right, the others mean nothing."""
    case = random_case(4, 32, 3, most=2, prompt_hi=200, heads=4, kv=2, dim=64).device()
    want = attention64(case, 0.125)
    true = share(case)
    lone = torch.tensor([t for s in range(32) if int(true.place[s]) < 0 for t in range(case.start[s], case.start[s + 1])])
    rng = np.random.default_rng(0)
    for _ in range(6):
        sh = share(case)
        for t in (sh.groups, sh.rows, sh.counts, sh.own, sh.place):
            flat = t.view(-1)
            keep = flat <= 0 if t is sh.own else flat < 0 if t is sh.place else torch.zeros_like(flat, dtype=torch.bool)
            wild = torch.from_numpy(rng.choice([-2 ** 31, -1, 0, 1, 5, 100, 10 ** 6, 2 ** 31 - 1], flat.numel()).astype(np.int32)).cuda()
            if t is sh.rows:                         # rows that any list names are written by it
                wild = torch.where(flat < 0, flat, flat[torch.from_numpy(rng.integers(0, max(1, int((flat >= 0).sum())), flat.numel())).cuda()])
            flat.copy_(torch.where(keep, flat, wild))
        sh.counts[1] = min(max(int(sh.counts[1]), 0), int((sh.rows >= 0).sum()))
        out, _ = attend_shared(case, sh, 0.125)
        err = (out.double().cpu() - want[0]).abs()[lone]
        assert (err <= want[2][lone] * (1.02 * 2.0 ** -7) + 1e-37).all()
    torch.cuda.synchronize()


def test_a_graph_of_both_calls_replayed_with_other_lengths():
    case = random_case(31, 40, 3, prompt_hi=300, own_hi=30, heads=8, kv=2, dim=64).device()
    sh = L.KvShared(40, case.T)
    out = torch.empty((case.T, 512), dtype=torch.bfloat16, device="cuda")
    ws = torch.empty(max(256, L.lora_kv_attention_shared_ws_bytes(case.cache, case.batch, sh, 8)), dtype=torch.uint8, device="cuda")

    def both():
        L.lora_kv_share(case.cache, case.batch, sh)
        L.lora_kv_attention_shared(case.cache, 0, case.batch, sh, case.qd, 512, 8, out, 512, None, 0.125, ws)

    both()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    lens = case.batch.seq_len.clone()
    for cut in (0, 1, 20, 0):
        case.batch.seq_len.copy_((lens - cut).clamp(min=1))
        case.lens = case.batch.seq_len.tolist()
        out.fill_(9.0)
        graph.replay()
        torch.cuda.synchronize()
        check_attention(case, (out, None), attention64(case, 0.125))


def test_on_another_stream():
    case = random_case(41, 30, 3, prompt_hi=300, heads=8, kv=2, dim=64).device()
    sh = share(case)
    want = attend_shared(case, sh, 0.125)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    out = torch.zeros_like(want[0])
    ws = torch.zeros(L.lora_kv_attention_shared_ws_bytes(case.cache, case.batch, sh, 8), dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    L.lora_kv_attention_shared(case.cache, 0, case.batch, sh, case.qd, 512, 8, out, 512, None, 0.125, ws, stream=side)
    side.synchronize()
    assert torch.equal(out, want[0])


def test_two_calls_at_once_on_two_streams():
    """Each with a workspace and results of its own; both kinds of tiles, cut ones among them."""
    cases = [random_case(43, 60, 2, most=3, prompt_hi=2500, own_hi=60, heads=8, kv=2, dim=64).device(),
             SharedCase([0] * 50, [3000], [7] * 50, [1] * 50, heads=32, kv=8, dim=128, seed=3).device()]
    shares = [share(c) for c in cases]
    want = [attend_shared(c, sh, 0.125)[0] for c, sh in zip(cases, shares)]
    outs = [torch.zeros_like(w) for w in want]
    wss = [torch.empty(L.lora_kv_attention_shared_ws_bytes(c.cache, c.batch, sh, c.heads), dtype=torch.uint8, device="cuda") for c, sh in zip(cases, shares)]
    streams = [torch.cuda.Stream() for _ in cases]
    torch.cuda.synchronize()
    for _ in range(10):
        for c, sh, out, ws, st in zip(cases, shares, outs, wss, streams):
            L.lora_kv_share(c.cache, c.batch, sh, stream=st)
            L.lora_kv_attention_shared(c.cache, 0, c.batch, sh, c.qd, c.qd.stride(0), c.heads, out, out.shape[1], None, 0.125, ws, stream=st)
    torch.cuda.synchronize()
    for out, w in zip(outs, want):
        assert torch.equal(out, w)


# Groups of more than 32 rows x heads that share K go in long tiles where all of them together are enough work: rows x group x shared tokens x
# key/value heads above 2.8e6 of such groups
@pytest.mark.parametrize("heads,kv,dim,width,tokens", [
    (32, 8, 128, 70, 2000), (16, 8, 64, 100, 2000), (8, 8, 40, 100, 4000), (20, 5, 80, 90, 2100), (8, 4, 256, 100, 4003), (64, 1, 64, 30, 2000), (6, 2, 8, 250, 2000)])
@pytest.mark.parametrize("causal", [True, False])
def test_groups_in_long_tiles(heads, kv, dim, width, tokens, causal):
    assert width * heads * tokens > 2.9e6            # rows x group x heads of K and V: rows x heads
    rng = np.random.default_rng(width)
    case = SharedCase([0] * width + [-1, -1], [tokens], [int(i) for i in rng.integers(0, 60, width + 2)], [1] * (width - 1) + [5, 1, 3], heads=heads, kv=kv, dim=dim, seed=dim)
    check(case, causal=causal)


@pytest.mark.parametrize("seqs,prompts,most,prompt_hi", [(300, 2, 1, 4000), (60, 3, 8, 4000), (500, 9, 1, 2000), (40, 1, 40, 2500)])
def test_long_tiles_among_others(seqs, prompts, most, prompt_hi):
    """Plans in LDS and in memory, groups in both kinds of tiles, rows of their own in long ones as well."""
    check(random_case(seqs + most, seqs, prompts, most=most, prompt_hi=prompt_hi, own_hi=60, heads=16, kv=4, dim=64))


def test_a_graph_whose_groups_change_their_tiles():
    """Lengths on both sides of the rule for groups' tiles, in one captured call."""
    width = 70
    case = SharedCase([0] * width, [3000], [i % 9 for i in range(width)], [1] * width, heads=32, kv=8, dim=64, seed=6).device()
    sh = L.KvShared(width, case.T)
    out = torch.empty((case.T, 2048), dtype=torch.bfloat16, device="cuda")
    ws = torch.empty(L.lora_kv_attention_shared_ws_bytes(case.cache, case.batch, sh, 32), dtype=torch.uint8, device="cuda")

    def both():
        L.lora_kv_share(case.cache, case.batch, sh)
        L.lora_kv_attention_shared(case.cache, 0, case.batch, sh, case.qd, 2048, 32, out, 2048, None, 0.125, ws)

    both()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    lens = case.batch.seq_len.clone()
    for most in (4000, 700, 2990, 40, 4000):         # 70 x 32 x 1250 is the border
        case.batch.seq_len.copy_(lens.clamp(max=most))
        case.lens = case.batch.seq_len.tolist()
        out.fill_(9.0)
        graph.replay()
        torch.cuda.synchronize()
        check_attention(case, (out, None), attention64(case, 0.125))


def test_untrue_groups_in_long_tiles_stay_within_bounds():
    """As above, with groups whose rows and tokens are as many as the batch has room for."""
    case = SharedCase([0] * 60 + [-1] * 4, [3000], [5] * 64, [1] * 64, heads=16, kv=4, dim=64, seed=9).device()
    want = attention64(case, 0.125)
    lone = torch.arange(60, 64)
    rng = np.random.default_rng(1)
    for _ in range(6):
        sh = share(case)
        n = int((sh.rows >= 0).sum())
        wild = rng.choice([-2 ** 31, -1, 0, 7, 60, 3000, 10 ** 6, 2 ** 31 - 1], sh.groups.numel()).astype(np.int32)
        wild.reshape(-1, 4)[0] = [int(rng.integers(0, 64)), int(rng.choice([2992, 3008, 10 ** 6])), int(rng.integers(0, 9)), int(rng.choice([60, 64, 10 ** 6]))]
        sh.groups.view(-1).copy_(torch.from_numpy(wild).cuda())
        sh.rows[:n] = sh.rows[torch.from_numpy(rng.integers(0, n, n)).cuda()]
        sh.own[:60] = torch.from_numpy(rng.choice([1, 16, 2992, 2 ** 31 - 1], 60).astype(np.int32)).cuda()
        sh.place[:60] = torch.from_numpy(rng.choice([0, 59, 63, 2 ** 31 - 1], 60).astype(np.int32)).cuda()
        out, _ = attend_shared(case, sh, 0.125)
        err = (out.double().cpu() - want[0]).abs()[lone]
        assert (err <= want[2][lone] * (1.02 * 2.0 ** -7) + 1e-37).all()
    torch.cuda.synchronize()
