"""Helpers of the tests of sequences that share pages (not a test module): batches whose prompts' whole pages are shared, and
the groups by their definition."""
from __future__ import annotations

import numpy as np
import torch

import paper_2604_07173_amd as L
from kv_common import KvCase


class SharedCase(KvCase):
    """Sequence s answers prompt of[s] (-1: none): the whole pages of its prompts[of[s]] tokens are those of all its answers; then
    come own[s] tokens and rows[s] new ones."""

    def __init__(self, of, prompts, own, rows, heads=4, kv=2, dim=64, page=16, slot_major=False, seed=0, stale=float("nan"), layers=1,
                 max_rows=None, v_scale=1.0, q_scale=1.5):
        rng = np.random.default_rng(seed)
        self.rows, self.heads, self.kv, self.dim, self.page = list(rows), heads, kv, dim, page
        self.slot_major, self.layers = slot_major, layers
        prompt = [prompts[o] if o >= 0 else 0 for o in of]
        self.lens = [p + m + r for p, m, r in zip(prompt, own, rows)]
        whole = [p // page for p in prompts]
        held = [-(-n // page) for n in self.lens]
        mine = [h - (whole[o] if o >= 0 else 0) for h, o in zip(held, of)]
        self.n_pages = sum(whole) + sum(mine) + 3
        order = rng.permutation(self.n_pages)
        first = np.concatenate([[0], np.cumsum(whole)])
        self.table = np.full((len(of), max([1] + held)), -7, np.int32)
        at = int(first[-1])
        for s, o in enumerate(of):
            w = whole[o] if o >= 0 else 0
            if w:
                self.table[s, :w] = order[first[o]:first[o] + w]
            self.table[s, w:held[s]] = order[at:at + mine[s]]
            at += mine[s]
        shape = (layers, self.n_pages, page, kv, dim) if slot_major else (layers, self.n_pages, kv, page, dim)
        self.kt, self.vt = (torch.full(shape, stale, dtype=torch.bfloat16) for _ in range(2))
        self.k5 = self.kt.transpose(2, 3) if slot_major else self.kt
        self.v5 = self.vt.transpose(2, 3) if slot_major else self.vt
        filled = np.zeros(self.n_pages, np.int64)
        for s, n in enumerate(self.lens):
            for c in range(held[s]):
                filled[self.table[s, c]] = max(filled[self.table[s, c]], min(page, n - c * page))
        for i in np.nonzero(filled)[0]:
            for t5, f in ((self.k5, 1.0), (self.v5, v_scale)):
                x = torch.from_numpy(rng.standard_normal((layers, kv, filled[i], dim)).astype(np.float32)) * f
                t5[:, i, :, :filled[i]] = x.to(torch.bfloat16)
        self.T = sum(rows)
        self.start = np.concatenate([[0], np.cumsum(rows)]).astype(np.int32)
        self.q = (q_scale * torch.from_numpy(rng.standard_normal((self.T, heads * dim)).astype(np.float32))).to(torch.bfloat16)
        self.max_rows = max([0] + list(rows)) if max_rows is None else max_rows


def random_case(seed, seqs, prompts, most=1, prompt_hi=300, own_hi=60, **kw):
    rng = np.random.default_rng(seed)
    of = rng.integers(-1, prompts, seqs)
    rows = np.ones(seqs, int) if most == 1 else rng.integers(0, most + 1, seqs)
    rows[rng.integers(seqs)] = most
    return SharedCase(of.tolist(), rng.integers(0, prompt_hi + 1, prompts).tolist(), rng.integers(0, own_hi + 1, seqs).tolist(), rows.tolist(),
                      seed=seed, **kw)


def groups_by_definition(table, lens, rows, page, min_pages=1, max_rows=0):
    """[(leader, shared tokens, members)] of a batch."""
    n = len(lens)
    whole = [max(0, lens[s] - rows[s]) // page for s in range(n)]
    part = [1 <= rows[s] and (not max_rows or rows[s] <= max_rows) and whole[s] >= min_pages for s in range(n)]
    groups = []
    for lead in range(n):
        key = lambda s: table[s][min_pages - 1]                                             # noqa: E731
        if not part[lead] or any(part[s] and key(s) == key(lead) for s in range(lead)):
            continue
        members, least = [], None
        for s in range(lead, n):
            if not part[s] or key(s) != key(lead):
                continue
            c = 0
            while c < min(whole[s], whole[lead]) and table[s][c] == table[lead][c]:
                c += 1
            if c >= min_pages:
                members.append(s)
                least = c if least is None else min(least, c)
        if len(members) >= 2:
            groups.append((lead, least * page, members))
    return groups


def expected_share(table, lens, rows, start, page, room, **kw):
    """What lora_kv_share writes, as lists."""
    n = len(lens)
    found = groups_by_definition(table, lens, rows, page, **kw)
    groups, listed, own, place = [], [], [0] * n, [-1] * n
    for lead, tokens, members in found:
        groups.append([lead, tokens, len(listed), sum(rows[s] for s in members)])
        for s in members:
            own[s], place[s] = tokens, len(listed)
            listed += range(start[s], start[s] + rows[s])
    counts = [len(found), len(listed), sum(len(m) for _, _, m in found), min(2 ** 31 - 1, sum((len(m) - 1) * t for _, t, m in found))]
    groups += [[-1, 0, 0, 0]] * (max(n // 2, 1) - len(groups))
    return dict(groups=groups, rows=listed + [-1] * (room - len(listed)), own=own, place=place, counts=counts)


def share(case, min_pages=1, max_rows=0, room=None, max_group_rows=0, stream=None):
    n = len(case.lens)
    sh = L.KvShared(n, case.T if room is None else room, max_group_rows)
    for t in (sh.groups, sh.rows, sh.own, sh.place, sh.counts, sh.ws):
        t.fill_(77)                                  # the call writes all of them
    L.lora_kv_share(case.cache, case.batch, sh, min_pages, max_rows, stream=stream)
    return sh


def attend_shared(case, sh, scale, causal=True, layer=0, lse=True, ldo=None, stream=None):
    ldo = ldo or case.heads * case.dim
    out = torch.full((case.T, ldo), 7.0, dtype=torch.bfloat16, device="cuda")
    e = torch.full((case.T, case.heads), 7.0, device="cuda") if lse else None
    ws = torch.empty(max(256, L.lora_kv_attention_shared_ws_bytes(case.cache, case.batch, sh, case.heads)), dtype=torch.uint8, device="cuda")
    ws.fill_(0xFF)                                   # a workspace holds anything, NaN here
    L.lora_kv_attention_shared(case.cache, layer, case.batch, sh, case.qd, case.qd.stride(0), case.heads, out, ldo, e, scale, ws,
                               causal=causal, stream=stream)
    return out, e
