"""Helpers of the paged cache's GPU tests (not a test module): batches with their tables, the operators'
definitions in 64 bits on the CPU, and the bounds that the results are held to."""
from __future__ import annotations

import math

import numpy as np
import torch

import paper_2604_07173_amd as L


class KvCase:
    """Caches with everything that a sequence does not hold set to `stale`, tables in random page order."""

    def __init__(self, rows, lens, heads=4, kv=2, dim=64, page=16, slot_major=False, seed=0, stale=float("nan"), spare=3,
                 layers=1, max_rows=None, v_scale=1.0, q_scale=1.5, wide=0):
        rng = np.random.default_rng(seed)
        self.rows, self.lens, self.heads, self.kv, self.dim, self.page = list(rows), list(lens), heads, kv, dim, page
        held = [-(-n // page) for n in lens]
        self.n_pages = sum(held) + spare
        order = rng.permutation(self.n_pages)
        width = max([1] + held)
        self.table = np.full((len(lens), width), -7, np.int32)        # entries past the pages in use are never looked at
        at = 0
        for s, h in enumerate(held):
            self.table[s, :h] = order[at:at + h]
            at += h
        shape = (layers, self.n_pages, page, kv, dim) if slot_major else (layers, self.n_pages, kv, page, dim)
        self.kt, self.vt = (torch.full(shape, stale, dtype=torch.bfloat16) for _ in range(2))
        self.k5 = self.kt.transpose(2, 3) if slot_major else self.kt
        self.v5 = self.vt.transpose(2, 3) if slot_major else self.vt
        self.slot_major, self.layers = slot_major, layers
        for s, n in enumerate(lens):
            for c in range(held[s]):
                m = min(page, n - c * page)
                for t5, f in ((self.k5, 1.0), (self.v5, v_scale)):
                    x = torch.from_numpy(rng.standard_normal((layers, kv, m, dim)).astype(np.float32)) * f
                    t5[:, self.table[s, c], :, :m] = x.to(torch.bfloat16)
        T = sum(rows)
        self.T = T
        self.start = np.concatenate([[0], np.cumsum(rows)]).astype(np.int32)
        self.q = (q_scale * torch.from_numpy(rng.standard_normal((T, heads * dim + wide)).astype(np.float32))).to(torch.bfloat16)
        self.max_rows = max([0] + list(rows)) if max_rows is None else max_rows

    def device(self):
        self.kd, self.vd = self.kt.cuda(), self.vt.cuda()
        k, v = (t.transpose(2, 3) if self.slot_major else t for t in (self.kd, self.vd))
        self.cache = L.KvCache(k, v)
        self.batch = L.KvBatch(torch.from_numpy(self.start).cuda(), torch.tensor(self.lens, dtype=torch.int32).cuda(),
                               torch.from_numpy(self.table).cuda(), n_rows=self.T, max_rows=self.max_rows)
        self.qd = self.q.cuda()
        return self

    def tokens(self, s, layer=0):
        """K and V of a sequence in 64 bits: [kv][token][dim]."""
        n = self.lens[s]
        pages = self.table[s, :-(-n // self.page)].astype(np.int64)
        out = []
        for t5 in (self.k5, self.v5):
            x = t5[layer, pages].transpose(0, 1).reshape(self.kv, -1, self.dim)[:, :n]
            out.append(x.double())
        return out


def attention64(case, scale, causal=True, window=0, layer=0):
    """out, lse and the sum of the softmax weights times |v|, in 64 bits, row by row from the definition."""
    H, D, G = case.heads, case.dim, case.heads // case.kv
    out = torch.zeros((case.T, H, D), dtype=torch.float64)
    mag = torch.zeros_like(out)
    lse = torch.full((case.T, H), -math.inf, dtype=torch.float64)
    big = torch.zeros((case.T, H), dtype=torch.float64)
    for s, (r, n) in enumerate(zip(case.rows, case.lens)):
        if r == 0 or n == 0:
            continue
        k, v = case.tokens(s, layer)
        for i in range(r):
            pos, t = n - r + i, int(case.start[s]) + i
            hi = max(0, min(n, pos + 1)) if causal else n
            lo = max(0, pos - window + 1) if window else 0
            if lo >= hi:
                continue
            q = case.q[t, :H * D].double().view(case.kv, G, D)
            sc = torch.matmul(q, k[:, lo:hi].transpose(1, 2)) * scale
            m = sc.amax(-1, keepdim=True)
            p = (sc - m).exp()
            total = p.sum(-1, keepdim=True)
            out[t] = (torch.matmul(p, v[:, lo:hi]) / total).reshape(H, D)
            mag[t] = (torch.matmul(p, v[:, lo:hi].abs()) / total).reshape(H, D)
            lse[t] = (m + total.log()).reshape(H)
            big[t] = (torch.matmul(q.abs(), k[:, lo:hi].abs().transpose(1, 2)) * scale).amax(-1).reshape(H)
    return out.view(case.T, H * D), lse, mag.view(case.T, H * D), big


def attend(case, scale, causal=True, window=0, layer=0, lse=True, ldo=None, stream=None):
    ldo = ldo or case.heads * case.dim
    out = torch.full((case.T, ldo), 7.0, dtype=torch.bfloat16, device="cuda")
    e = torch.full((case.T, case.heads), 7.0, device="cuda") if lse else None
    ws = torch.empty(max(256, L.lora_kv_attention_ws_bytes(case.cache, case.batch, case.heads)), dtype=torch.uint8, device="cuda")
    ws.fill_(0xFF)                                                    # a workspace holds anything, NaN here
    L.lora_kv_attention(case.cache, layer, case.batch, case.qd, case.qd.stride(0), case.heads, out, ldo, e, scale, ws,
                        causal=causal, window=window, stream=stream)
    return out, e


def check_attention(case, got, want, what=""):
    """Every element of out within 2^-7 of the softmax-weighted |v|, twice the bound of one rounding to bf16 (8 significant
    bits, so half a step is at most 2^-8 of the value): the weights are rounded (at most 2^-8 of each), and so is the
    sum (2^-8 of it, and |sum| <= sum of |.|); 2 % more for the sums' own fp32 errors.  lse: fp32 sums of `dim` products and one logarithm, 2^-24 * dim of the sum of magnitudes and
    2^-20 of itself."""
    out, lse = got
    ref, ref_lse, mag, big = want
    W = case.heads * case.dim
    got64 = out[:, :W].double().cpu()
    bound = mag * (1.02 * 2.0 ** -7) + 1e-37
    err = (got64 - ref).abs()
    assert torch.isfinite(got64).all(), f"{what}: not finite at {torch.nonzero(~torch.isfinite(got64))[:4].tolist()}"
    assert (err <= bound).all(), f"{what}: {int((err > bound).sum())} beyond the bound, worst {float((err / bound).max()):.2f}"
    if lse is not None:
        e = lse.double().cpu()
        empty = torch.isinf(ref_lse)
        assert torch.equal(torch.isinf(e) & (e < 0), empty), f"{what}: rows without a token"
        tol = (2.0 ** -24 * case.dim * big + 2.0 ** -20 * (1 + ref_lse.abs()))[~empty]
        err = (e[~empty] - ref_lse[~empty]).abs()
        assert (err <= tol).all(), f"{what}: lse, worst {float((err / tol).max()):.2f}"
    assert int(case.batch.status.item()) == 0
