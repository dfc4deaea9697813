"""Append, attention and copies over caches whose layers, pages, heads and tokens lie in every order."""
import itertools

import numpy as np
import pytest
import torch

import paper_2604_07173_amd as L
from kv_common import KvCase, attend, attention64, check_attention

pytestmark = pytest.mark.gpu
ORDERS = list(itertools.permutations("lpht"))


def laid_out(t, order, hole=0):
    """The same values as t [layer][page][head][token][width], with dimensions in memory in `order`."""
    at = ["lpht".index(c) for c in order]
    shape = [t.shape[i] for i in at]
    shape[-1] += hole
    base = torch.full((*shape, t.shape[4]), 3.0, dtype=t.dtype, device=t.device)
    seen = base[:, :, :, :t.shape[at[3]]].permute(*(at.index(i) for i in range(4)), 4)
    seen.copy_(t)
    return seen


@pytest.mark.parametrize("order", ORDERS, ids="".join)
@pytest.mark.parametrize("hole", [0, 1])
def test_every_order(order, hole):
    case = KvCase([1, 5, 40], [30, 70, 61], 4, 2, 64, layers=2, seed=3, stale=5.0).device()
    case.cache = L.KvCache(*(laid_out(t, order, hole) for t in (case.kd, case.vd)))
    for layer in range(2):
        check_attention(case, attend(case, 0.125, layer=layer), attention64(case, 0.125, layer=layer))
    # the append, against the one into the plain order
    x = torch.randn((46, 8 * 64), device="cuda").bfloat16()
    plain = L.KvCache(case.kd, case.vd)
    rope = L.Rope(64)
    for cache in (case.cache, plain):
        L.lora_rope_append(cache, 1, case.batch, rope, None, 0, x[:, :128], 512, x[:, 128:], 512, None, 0, 0)
    torch.cuda.synchronize()
    assert torch.equal(case.cache.k, plain.k) and torch.equal(case.cache.v, plain.v)
    # and the copies
    moves = L.KvMoves(case.n_pages, 4)
    pairs = [(3, 0), (9, 2), (3, 8)]
    moves.pairs[:3] = torch.tensor(pairs, dtype=torch.int32)
    moves.counts[1] = 3
    want = [t.clone() for t in (plain.k, plain.v)]
    for w in want:
        for a, b in pairs:
            w[:, b] = w[:, a]
    L.lora_kv_copy_pages(case.cache, moves, max_moves=3)
    torch.cuda.synchronize()
    assert torch.equal(case.cache.k, want[0]) and torch.equal(case.cache.v, want[1])
    if hole:                                       # what lies between is left alone
        base = case.cache.k._base
        assert (base[:, :, :, -1] == 3.0).all()


def test_heads_outside_pages_at_offsets_beyond_32_bits():
    kv, page, dim = 2, 16, 128
    n_pages = (1 << 31) // (page * dim) + 8        # a head's pages alone pass 2^31 elements
    k, v = (torch.empty((1, kv, n_pages, page, dim), dtype=torch.bfloat16, device="cuda").transpose(1, 2) for _ in range(2))
    small = KvCase([1, 50], [100, 70], 4, kv, dim, seed=18).device()
    far = torch.from_numpy(small.table.astype(np.int64)).cuda() + (n_pages - small.n_pages)
    k[0, n_pages - small.n_pages:], v[0, n_pages - small.n_pages:] = small.kd[0], small.vd[0]
    want = attend(small, 0.1)
    small.cache = L.KvCache(k, v)
    small.batch = L.KvBatch(small.batch.row_start, small.batch.seq_len, far.int().contiguous(), small.T, max_rows=50)
    got = attend(small, 0.1)
    assert torch.equal(want[0], got[0]) and torch.equal(want[1], got[1])
