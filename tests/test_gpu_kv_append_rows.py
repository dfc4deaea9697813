"""lora_rope_append where the batch's row_start is no partition of its rows: a row that belongs to no sequence, or to another
place than the sequence's new rows, is not written."""
import pytest
import torch

import paper_2604_07173_amd as L
from kv_common import KvCase

pytestmark = pytest.mark.gpu


# sequences of 4, 3 and 5 new rows in lengths of 20, 19 and 30, in pages of 16: (row_start, rows that have a sequence)
@pytest.mark.parametrize("start,there", [
    ([0, 4, 7, 9], range(9)),               # the last three rows are nobody's
    ([2, 4, 7, 12], range(2, 12)),          # the first two neither
    ([0, 4, 7, 7], range(7)),
    ([0, 0, 0, 0], range(0)),
    ([12, 12, 12, 12], range(0)),
    ([5, 5, 7, 12], range(5, 12)),
])
@pytest.mark.parametrize("position", [False, True])
def test_rows_of_no_sequence_are_not_written(start, there, position):
    lens, kv, dim, page = [20, 19, 30], 2, 64, 16
    case = KvCase([4, 3, 5], lens, 4, kv, dim, page, stale=5.0, spare=6).device()
    table = torch.full((3, 4), -1, dtype=torch.int32, device="cuda")
    table[:, :2] = case.batch.table                      # room for more tokens, in pages that are in the cache
    table[:, 2:] = torch.tensor([p for p in range(case.n_pages) if p not in case.table][:6], device="cuda").view(3, 2)
    pos = torch.arange(12, dtype=torch.int32, device="cuda") if position else None
    batch = L.KvBatch(torch.tensor(start, dtype=torch.int32, device="cuda"), case.batch.seq_len, table, 12, position=pos)
    k = (torch.arange(12, device="cuda") + 100.0).bfloat16()[:, None].expand(12, kv * dim).contiguous()
    q = torch.ones((12, 4 * dim), dtype=torch.bfloat16, device="cuda")
    q_out = torch.zeros_like(q)
    want = case.kd.clone()
    for t in there:
        s = max(i for i in range(3) if start[i] <= t)
        p = lens[s] - start[s + 1] + t
        want[0, table[s, p // page], :, p % page] = 100.0 + t
    L.lora_rope_append(case.cache, 0, batch, None, q, 4 * dim, k, kv * dim, k, kv * dim, q_out, 4 * dim, 4)
    torch.cuda.synchronize()
    assert int(batch.status.item()) == L.LORA_STATUS_BAD_LENGTH
    assert torch.equal(case.kd, want)
    assert torch.equal(q_out, q)                         # q has no place to go wrong
