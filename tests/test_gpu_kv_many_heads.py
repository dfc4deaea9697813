"""Attention of the largest batches: as many rows x heads as a call takes, where a workgroup for every sequence and head would be more than
a launch may have.  Every sequence has one token, so that each row's result is that token's V."""
import pytest
import torch

import paper_2604_07173_amd as L

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n_seqs,rows,heads,max_rows", [
    (262144, 1, 64, 0),           # one row each, the longest chunk unknown
    (262144, 1, 64, 1),
    (31775, 33, 512, 33),         # as many in all, by a row too many for short tiles
])
def test_every_row_of_the_largest_batches(n_seqs, rows, heads, max_rows):
    dim, n_pages = 8, 1000
    k, v = (torch.randn((1, n_pages, heads, 1, dim), device="cuda").bfloat16() for _ in range(2))
    cache = L.KvCache(k, v)
    table = torch.randint(0, n_pages, (n_seqs, 1), dtype=torch.int32, device="cuda")
    length = torch.ones(n_seqs, dtype=torch.int32, device="cuda")
    length[::7] = 0
    start = torch.arange(n_seqs + 1, dtype=torch.int32, device="cuda") * rows
    T = n_seqs * rows
    batch = L.KvBatch(start, length, table, T, max_rows)
    q = torch.randn((T, heads * dim), device="cuda", dtype=torch.bfloat16)
    out = torch.full_like(q, 7.0)
    ws = torch.empty(L.lora_kv_attention_ws_bytes(cache, batch, heads), dtype=torch.uint8, device="cuda")
    L.lora_kv_attention(cache, 0, batch, q, heads * dim, heads, out, heads * dim, None, 0.3, ws, causal=False)
    torch.cuda.synchronize()
    assert int(batch.status.item()) == 0
    want = v[0, :, :, 0][table[:, 0].long()]
    want[::7] = 0.0
    assert (out.view(n_seqs, rows, heads, dim) == want[:, None]).all()
