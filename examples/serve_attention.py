"""A serving loop around the attention block of a dense LLM whose users bring their own adapters: base products,
LoRA updates of q, k, v and o, rotary positions, a paged cache and attention over it, with prompts in
chunks beside decoding users, forks, sequences that end, and a compaction.

    python examples/serve_attention.py [--steps 12] [--check] [--answers 5]

Every step is the same few calls for all users together:
    lora_kv_plan, lora_kv_copy_pages        who continues what, and room for the new rows
    per layer:  x Wqkv                      the base product (torch)
                lora_build_apply_group      += scale x A B of every row's own adapter, for q, k and v
                lora_rope_append            q rotated, k rotated into its page, v into its page
                lora_kv_attention           new rows over all of their sequence
                lora_apply                  the output projection's update on top of its base product
--answers N draws N answers to each of a few prompts instead, token by token: the prompts fork, and every step is
    lora_kv_plan, lora_kv_copy_pages, lora_kv_share
    per layer:  lora_add_norm                   the residual stream takes the layer before, and is normalised for the next products
                base products, LoRA updates and lora_rope_append as above
                lora_kv_attention_shared        a prompt's pages are read once for all of its answers
    lora_add_norm, the product with the vocabulary, lora_sample
--check recomputes every sequence from its first token in 64 bits, exactly and with the loop's roundings to bf16, and
compares how far the loop and the rounded recomputation are from the exact one.
"""
from __future__ import annotations

import argparse
import math
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2604_07173_amd as L                                                   # noqa: E402


class Layers:
    """Base weights and adapters of a few attention blocks (random)."""

    def __init__(self, n_layers=2, hidden=512, heads=8, kv=2, dim=64, adapters=5, rank=16, seed=0):
        g = torch.Generator().manual_seed(seed)
        self.n_layers, self.hidden, self.heads, self.kv, self.dim = n_layers, hidden, heads, kv, dim
        self.widths = [heads * dim, kv * dim, kv * dim]
        rand = lambda *s: (torch.randn(s, generator=g) / math.sqrt(s[0])).to(torch.bfloat16)      # noqa: E731
        self.wqkv = [rand(hidden, sum(self.widths)).cuda() for _ in range(n_layers)]
        self.wo = [rand(heads * dim, hidden).cuda() for _ in range(n_layers)]
        projs = [(hidden, w) for w in self.widths] + [(heads * dim, hidden)]
        self.scale = [0.5 + 0.25 * a for a in range(adapters)]
        desc = L.PoolDesc(adapters, n_layers, 1, projs, rank, scale=self.scale)
        self.pool = L.lora_register_pool(desc, torch.empty(L.lora_pool_bytes(desc), dtype=torch.uint8, device="cuda"))
        self.ab = {}
        for a in range(adapters):
            for layer in range(n_layers):
                pairs = [(rand(i, rank), rand(rank, o)) for i, o in projs]
                self.ab[a, layer] = pairs
                L.lora_pool_load_adapter_layer(self.pool, a, layer, torch.cat([m.flatten() for p in pairs for m in p]).cuda())
        torch.cuda.synchronize()


class Server:
    """Sequences in slots over one paged cache; step() takes them all forward."""

    def __init__(self, model: Layers, slots=16, n_pages=400, page=16, max_len=512):
        m = self.model = model
        shape = (m.n_layers, n_pages, m.kv, page, m.dim)
        self.cache = L.KvCache(*(torch.zeros(shape, dtype=torch.bfloat16, device="cuda") for _ in range(2)))
        i32 = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")                         # noqa: E731
        # two states, so that a step's tables are made while the step before may still be reading its own
        self.states = [L.KvState(i32(slots, max_len // page) - 1, i32(slots), i32(n_pages)) for _ in range(2)]
        self.moves = L.KvMoves(n_pages, slots)
        self.rope = L.Rope(m.dim, scaling=L.LORA_ROPE_PARTS, factor=4.0, original_len=128.0, low=1.0, high=8.0)
        self.slots, self.n_pages = slots, n_pages
        self.length = [0] * slots
        self.adapter = [-1] * slots

    def plan(self, src, new_len):
        """Slot s goes on from slot src[s], new_len[s] tokens long (0: it ends)."""
        now, to = self.states
        dev = lambda v: torch.tensor(v, dtype=torch.int32).cuda()                                 # noqa: E731
        L.lora_kv_plan(self.cache, now, to, dev(src), dev(new_len), self.moves)
        L.lora_kv_copy_pages(self.cache, self.moves, max_moves=self.slots)
        self.states = [to, now]
        self.length = list(new_len)
        self.adapter = [self.adapter[p] if p >= 0 else -1 for p in src]

    def compact(self):
        now, to = self.states
        L.lora_kv_compact(self.cache, now, to, self.moves)
        L.lora_kv_copy_pages(self.cache, self.moves, max_moves=self.n_pages // 2)
        self.states = [to, now]

    def forward(self, x, rows):
        """x: the new rows' inputs, slot after slot, rows[s] of slot s.  Returns the last layer's rows."""
        m, P, state = self.model, x.shape[0], self.states[0]
        start = torch.from_numpy(np.concatenate([[0], np.cumsum(rows)]).astype(np.int32)).cuda()
        batch = L.KvBatch(start, state.seq_len, state.table, n_rows=P, max_rows=max(rows))
        ids = torch.from_numpy(np.repeat(self.adapter, rows).astype(np.int32)).cuda()
        seg = L.Segments(P)
        ws = torch.empty(max(L.lora_group_ws_bytes(m.pool, 0, 3, P), L.lora_v_bytes(m.pool, 3, P), 256), dtype=torch.uint8, device="cuda")
        aws = torch.empty(L.lora_kv_attention_ws_bytes(self.cache, batch, m.heads), dtype=torch.uint8, device="cuda")
        wq, wk, _ = m.widths
        for layer in range(m.n_layers):
            qkv = x @ m.wqkv[layer]
            q, k, v = qkv, qkv[:, wq:], qkv[:, wq + wk:]
            ld = qkv.shape[1]
            if layer == 0:
                L.lora_build_apply_group(m.pool, 0, 0, x, m.hidden, None, ids, None, P, seg, [q, k, v], [ld] * 3, ws)
            else:
                L.lora_apply_group(m.pool, layer, 0, x, m.hidden, None, seg, [q, k, v], [ld] * 3, ws)
            L.lora_rope_append(self.cache, layer, batch, self.rope, q, ld, k, ld, v, ld, q, ld, m.heads)     # q in place
            out = torch.empty((P, wq), dtype=torch.bfloat16, device="cuda")
            L.lora_kv_attention(self.cache, layer, batch, q, ld, m.heads, out, wq, None, 1.0 / math.sqrt(m.dim), aws)
            y = out @ m.wo[layer]
            L.lora_apply(m.pool, layer, 3, out, wq, None, seg, y, m.hidden, ws)
            x = x + y
        self.status = batch.status
        return x


class Answers(Server):
    """A server that draws tokens: slots 0 .. prompts - 1 hold the prompts, the others their answers."""

    def __init__(self, model: Layers, vocab=1003, seed=0, **kw):
        super().__init__(model, **kw)
        g = torch.Generator().manual_seed(seed + 1)
        m, rand = model, lambda *s: torch.randn(s, generator=g)                                   # noqa: E731
        self.vocab = vocab
        self.embed = rand(vocab, m.hidden).to(torch.bfloat16).cuda()
        self.head = (rand(m.hidden, vocab) * (3.0 / math.sqrt(m.hidden))).to(torch.bfloat16).cuda()
        self.gains = [(1.0 + 0.2 * rand(m.hidden)).to(torch.bfloat16).cuda() for _ in range(m.n_layers + 1)]
        self.norms = [L.Norm(w, eps=1e-6) for w in self.gains]

    def logits(self, tokens, rows):
        """tokens: the new ones, slot after slot, rows[s] of slot s, on the device.  Logits of every such slot's last row."""
        m, P, state = self.model, tokens.shape[0], self.states[0]
        start = torch.from_numpy(np.concatenate([[0], np.cumsum(rows)]).astype(np.int32)).cuda()
        batch = L.KvBatch(start, state.seq_len, state.table, n_rows=P, max_rows=max(rows))
        # rows of groups: 16 a sequence at most take part, and the attention's workspace has two results for each
        shared = L.KvShared(self.slots, min(P, 16 * self.slots))
        L.lora_kv_share(self.cache, batch, shared, max_rows=16)
        ids = torch.from_numpy(np.repeat(self.adapter, rows).astype(np.int32)).cuda()
        seg = L.Segments(P)
        ws = torch.empty(max(L.lora_group_ws_bytes(m.pool, 0, 3, P), L.lora_v_bytes(m.pool, 3, P), 256), dtype=torch.uint8, device="cuda")
        aws = torch.empty(L.lora_kv_attention_shared_ws_bytes(self.cache, batch, shared, m.heads), dtype=torch.uint8, device="cuda")
        wq, wk, _ = m.widths
        h, y, x = self.embed[tokens.long()], None, torch.empty((P, m.hidden), dtype=torch.bfloat16, device="cuda")
        for layer in range(m.n_layers):
            L.lora_add_norm(self.norms[layer], P, h, m.hidden, y, m.hidden, h, m.hidden, x, m.hidden)      # h += y in place
            qkv = x @ m.wqkv[layer]
            q, k, v = qkv, qkv[:, wq:], qkv[:, wq + wk:]
            ld = qkv.shape[1]
            if layer == 0:
                L.lora_build_apply_group(m.pool, 0, 0, x, m.hidden, None, ids, None, P, seg, [q, k, v], [ld] * 3, ws)
            else:
                L.lora_apply_group(m.pool, layer, 0, x, m.hidden, None, seg, [q, k, v], [ld] * 3, ws)
            L.lora_rope_append(self.cache, layer, batch, self.rope, q, ld, k, ld, v, ld, q, ld, m.heads)
            out = torch.empty((P, wq), dtype=torch.bfloat16, device="cuda")
            L.lora_kv_attention_shared(self.cache, layer, batch, shared, q, ld, m.heads, out, wq, None, 1.0 / math.sqrt(m.dim), aws)
            y = out @ m.wo[layer]
            L.lora_apply(m.pool, layer, 3, out, wq, None, seg, y, m.hidden, ws)
        L.lora_add_norm(self.norms[-1], P, h, m.hidden, y, m.hidden, None, 0, x, m.hidden)
        self.status, self.spared = batch.status, shared.counts
        last = (start[1:] - 1)[start[1:] > start[:-1]].long()
        return x[last] @ self.head

    def draw(self, logits, how, u):
        token = torch.empty(logits.shape[0], dtype=torch.int32, device="cuda")
        L.lora_sample(logits, self.vocab, logits.shape[0], self.vocab, how, u, token, dtype=L.LORA_DTYPE_BF16)
        return token


def answer(prompts=3, width=5, steps=12, seed=0, check=False):
    """Draws `width` answers of `steps` tokens to each of a few prompts.  With check: the error of the logits as a multiple of what
    the roundings make, and for every draw the logits, the settings, the random numbers and the tokens."""
    rng = np.random.default_rng(seed)
    model = Layers(seed=seed)
    server = Answers(model, seed=seed, slots=prompts * (width + 1))
    slots, of = server.slots, [s % prompts for s in range(prompts * (width + 1))]
    text = [rng.integers(0, server.vocab, int(rng.integers(20, 150))).tolist() if s < prompts else [] for s in range(slots)]
    rows = [len(t) for t in text]
    server.plan([-1] * slots, rows)
    for s in range(prompts):
        server.adapter[s] = int(rng.integers(-1, 5))
    dev = lambda a, t: torch.from_numpy(np.asarray(a, t)).cuda()                                  # noqa: E731
    # the answers have temperatures and limits of their own
    n = slots - prompts
    settings = dict(temperature=rng.choice([0.0, 0.7, 1.0, 1.3], n), top_k=rng.choice([0, 40, 5], n), top_p=rng.choice([1.0, 0.9, 0.6], n), min_p=rng.choice([0.0, 0.05], n))
    how = L.Sampling(*(dev(settings[f], np.int32 if f == "top_k" else np.float32) for f in ("temperature", "top_k", "top_p", "min_p")))
    logits = server.logits(dev(sum(text, []), np.int64), rows)[dev([of[s] for s in range(prompts, slots)], np.int64)].contiguous()
    drawn, off, rounding = [], 0.0, 0.0
    for step in range(steps):
        u = rng.random(n).astype(np.float32)
        token = server.draw(logits, how, dev(u, np.float32))
        if check:
            drawn.append((logits.float().cpu().numpy(), settings, u, token.cpu().numpy()))
        # at first all answers fork from their prompts, which stay as they are
        src = [s if s < prompts or step else of[s] for s in range(slots)]
        before = [server.length[p] for p in src]
        server.plan(src, [b + (s >= prompts) for s, b in enumerate(before)])
        if step % 5 == 4:
            server.compact()
        logits = server.logits(token, [0] * prompts + [1] * n)
        for s, t in zip(range(prompts, slots), token.tolist()):
            text[s] = (text[of[s]] if step == 0 else text[s]) + [t]
        groups, _, members, spared = server.spared.tolist()
        assert int(server.moves.status) == 0 and int(server.status) == 0
        line = f"step {step}: {n} answers, {members} of them in {groups} groups, {spared} tokens read once less"
        if check:
            freq = L.lora_rope_freqs(model.dim, scaling=L.LORA_ROPE_PARTS, factor=4.0, original_len=128.0, low=1.0, high=8.0)
            for s in range(prompts, slots):
                x = server.embed.cpu()[text[s]]
                exact, same = (recompute(model, x, server.adapter[s], freq, rounded, server)[-1] for rounded in (False, True))
                got = logits[s - prompts].double().cpu()
                off += float((got - exact).square().sum())
                rounding += float((same - exact).square().sum())
            line += f", error {(off / rounding) ** 0.5:.2f} times what rounding to bf16 makes"
        print(line, flush=True)
    return ((off / rounding) ** 0.5 if rounding else 0.0), drawn


def recompute(model: Layers, x, adapter, freq, rounded: bool, answers=None):
    """One sequence from its first token, in 64 bits on the CPU; rounded: to bf16 wherever the loop above holds bf16.  answers: with its
    norms, and up to the logits."""
    m, r = model, (lambda t: t.to(torch.bfloat16).double()) if rounded else (lambda t: t)
    n = x.shape[0]
    turn = torch.polar(torch.ones(n, m.dim // 2, dtype=torch.float64), torch.arange(n).double()[:, None] * torch.tensor(freq, dtype=torch.float64))
    x = x.double()

    def lora(layer, j, inp):
        if adapter < 0:
            return 0.0
        a, b = model.ab[adapter, layer][j]
        return model.scale[adapter] * (inp @ a.double() @ b.double())

    def turned(t, heads):
        t = t.view(n, heads, 2, m.dim // 2)
        z = torch.complex(t[:, :, 0], t[:, :, 1]) * turn[:, None]
        return r(torch.stack([z.real, z.imag], 2).view(n, heads, m.dim))

    def norm(layer):
        if answers is None:
            return x
        return r(x / (x.square().mean(1, keepdim=True) + 1e-6).sqrt() * answers.gains[layer].cpu().double())

    for layer in range(m.n_layers):
        inp = norm(layer)
        qkv = torch.split(r(inp @ m.wqkv[layer].cpu().double()), m.widths, dim=1)
        q, k, v = (r(t + lora(layer, j, inp)) for j, t in enumerate(qkv))
        q, k, v = turned(q, m.heads), turned(k, m.kv), v.view(n, m.kv, m.dim)
        k, v = (t.repeat_interleave(m.heads // m.kv, 1).transpose(0, 1).contiguous() for t in (k, v))
        s = torch.matmul(q.transpose(0, 1), k.transpose(1, 2).contiguous()) / math.sqrt(m.dim)
        s = s.masked_fill(torch.ones(n, n, dtype=torch.bool).triu(1), -math.inf)
        out = r(torch.matmul(torch.softmax(s, -1), v).transpose(0, 1).reshape(n, -1))
        y = r(r(out @ m.wo[layer].cpu().double()) + lora(layer, 3, out))
        # (the last norm takes the sum as it is)
        x = x + y if answers is not None and layer == m.n_layers - 1 else r(x + y)
    return x if answers is None else r(norm(-1) @ answers.head.cpu().double())


def main(argv=None):
    """With --check: how many times what the roundings make the error is, and the worst row's share of error."""
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--steps", type=int, default=12)
    ap.add_argument("--check", action="store_true")
    ap.add_argument("--seed", type=int, default=0)
    ap.add_argument("--answers", type=int, default=0)
    args = ap.parse_args(argv)
    if args.answers:
        return answer(width=args.answers, steps=args.steps, seed=args.seed, check=args.check)[0], 0.0
    rng = np.random.default_rng(args.seed)
    model = Layers(seed=args.seed)
    server = Server(model)
    inputs = [torch.zeros(0, model.hidden, dtype=torch.bfloat16) for _ in range(server.slots)]     # of every sequence so far
    waiting = [0] * server.slots                       # prompt tokens that a sequence still has to take in
    worst, off, rounding = 0.0, 0.0, 0.0
    for step in range(args.steps):
        # the scheduler's decisions: who ends, who is new, who forks, and everybody's next rows
        src, rows = list(range(server.slots)), [0] * server.slots
        for s in range(server.slots):
            if server.length[s] and not waiting[s] and rng.random() < 0.12:
                server.length[s] = 0
                src[s] = -1
        idle = [s for s in range(server.slots) if server.length[s] == 0]
        ready = [s for s in range(server.slots) if server.length[s] and not waiting[s]]
        for s in idle:
            if ready and rng.random() < 0.2:            # another answer to the same prompt
                src[s] = int(rng.choice(ready))
                inputs[s] = inputs[src[s]]
                rows[s] = 1
            elif rng.random() < 0.5:
                src[s], inputs[s] = -1, inputs[s][:0]
                waiting[s] = int(rng.integers(1, 150))
        for s in range(server.slots):
            if waiting[s]:
                rows[s] = min(waiting[s], 64)           # a chunk of the prompt
                waiting[s] -= rows[s]
            elif src[s] == s and server.length[s]:
                rows[s] = 1
        if not sum(rows):
            continue
        before = [server.length[p] if p >= 0 else 0 for p in src]
        server.plan(src, [b + r for b, r in zip(before, rows)])
        for s in range(server.slots):
            if src[s] == -1 and rows[s]:
                server.adapter[s] = int(rng.integers(-1, 5))
        if step % 4 == 3:
            server.compact()
        new = [torch.from_numpy(rng.standard_normal((r, model.hidden)).astype(np.float32)).to(torch.bfloat16) for r in rows]
        out = server.forward(torch.cat(new).cuda(), rows)
        for s, r in enumerate(rows):
            inputs[s] = torch.cat([inputs[s], new[s]]) if server.length[s] else inputs[s][:0]
        torch.cuda.synchronize()
        used, _, free, _ = server.moves.counts.tolist()
        assert int(server.moves.status) == 0 and int(server.status) == 0
        line = f"step {step}: {sum(1 for r in rows if r)} sequences, {sum(rows)} rows, {used} pages in use, {free} free"
        if args.check:
            freq = L.lora_rope_freqs(model.dim, scaling=L.LORA_ROPE_PARTS, factor=4.0, original_len=128.0, low=1.0, high=8.0)
            at = 0
            for s, r in enumerate(rows):
                if r:
                    exact, same = (recompute(model, inputs[s], server.adapter[s], freq, rounded)[-r:] for rounded in (False, True))
                    got = out[at:at + r].double().cpu()
                    worst = max(worst, float(((got - exact).norm(dim=1) / exact.norm(dim=1)).max()))
                    off += float((got - exact).square().sum())
                    rounding += float((same - exact).square().sum())
                at += r
            line += f", error {(off / rounding) ** 0.5:.2f} times what rounding to bf16 makes, at most {worst:.3f} of a row"
        print(line, flush=True)
    return (off / rounding) ** 0.5 if rounding else 0.0, worst


if __name__ == "__main__":
    ratio, row = main()
    sys.exit(ratio > 2.0 or row > 0.5)
