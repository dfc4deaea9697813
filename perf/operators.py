"""Timed cases of the operators between the q/k/v and the output projection of an attention layer: rotary
positions with the append to a paged cache, attention of new rows over that cache, and the bookkeeping of
its pages.

A case is one call (for pages: the call and the data movement that it asks for).  `own` says who computes it:
False the plain form of this file, in torch operations of 32 bits that are rounded once at the end, True the
library's entry points.

Fields of a case:
  op          "append", "attend", "pages" (fork, free, truncate and extend) or "compact"
  seqs        sequences of the batch (pages, compact: sequence slots)
  rows        new rows of the batch (append, attend), shared out by `split`: "even", "ragged" (uneven, some
              sequences without a row) or "mixed" (one long chunk, one row for everybody else)
  ctx_lo, ctx_hi   tokens that a sequence has before its new rows, spread over the logarithm
  heads, kv, dim   query heads, key/value heads, width of a head
  page        tokens of a page;  slot_major: pages laid out [token][head] instead of [head][token]
  spare       share of the cache's pages that no sequence holds
  rot, pairing, scaling    append: rotated width of a head, "half" or "interleaved", "plain", "linear", "base" or "parts"
  f32         append: inputs in 32 bits (the sums of a base product and a delta) instead of bf16
  fused       append: q, k and v are column ranges of one buffer
  causal, window   attend: the mask;  lse: the logarithm of the softmax sum is asked for too
  layers      pages, compact: layers that share the tables
  width       pages: sequences that a fork makes of one;  done: share of the slots that end or fall back
  shape       seed of the lengths, which belong to the case and not to its inputs
"""
import math

import numpy as np
import torch

own = False

_DEFAULTS = dict(op="attend", seqs=1, rows=1, split="even", ctx_lo=0, ctx_hi=0, heads=32, kv=8, dim=128, page=16,
                 slot_major=False, spare=0.1, rot=128, pairing="half", scaling="plain", f32=False, fused=True,
                 causal=True, window=0, lse=False, layers=1, width=1, done=0.0, shape=1)


def _case(name=None, **kw):
    unknown = set(kw) - set(_DEFAULTS)
    if unknown:
        raise ValueError(f"unknown fields {sorted(unknown)}")
    c = dict(_DEFAULTS, **kw)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # a decode batch's q, k and v after their LoRA updates: one token for each of 64 users, far into long contexts
        _case("append_decode_64", op="append", seqs=64, rows=64, ctx_lo=1000, ctx_hi=30000, scaling="parts"),
        # an odd batch of prompt chunks: narrow heads rotated in part, neighbours paired, sums in 32 bits
        _case("append_odd_f32", op="append", seqs=7, rows=1333, split="ragged", ctx_lo=1, ctx_hi=5000, heads=12, kv=4, dim=80,
              rot=48, pairing="interleaved", scaling="linear", f32=True, page=8, slot_major=True),
        # the prefill workload's 8 requests of 2048 tokens
        _case("append_prefill_16384", op="append", seqs=8, rows=16384),
        # one user's next token: latency
        _case("attend_decode_1", seqs=1, rows=1, ctx_lo=1500, ctx_hi=1500),
        # the llama-shaped decode batch: 256 users with contexts of all lengths
        _case("attend_decode_256", seqs=256, rows=256, ctx_lo=100, ctx_hi=4000),
        # few users with very long contexts
        _case("attend_decode_long", seqs=3, rows=3, ctx_lo=60000, ctx_hi=130000, lse=True),
        # drafted tokens are verified: a few rows per sequence over a sliding window, odd heads
        _case("attend_verify_window", seqs=48, rows=230, split="ragged", ctx_lo=10, ctx_hi=9000, heads=20, kv=5, dim=80, page=8,
              window=1500, slot_major=True),
        # prefill of eight requests of 2048 tokens
        _case("attend_prefill_16384", seqs=8, rows=16384),
        # chunked prefill: a prompt's next chunk over what is cached of it, a decode token for 64 other users
        _case("attend_mixed_2048", seqs=65, rows=2048, split="mixed", ctx_lo=500, ctx_hi=16000),
        # one step of a small server: sequences end and grow, a few fork; one layer's pages
        _case("pages_step_64", op="pages", seqs=64, ctx_lo=10, ctx_hi=2000, width=1, done=0.1),
        # parallel sampling: prompts fork into eight sequences each, every one writes a page of its own
        _case("pages_fork_256", op="pages", seqs=256, ctx_lo=200, ctx_hi=2000, width=8, layers=16, done=0.05),
        # half of a cache's sequences have gone: the pages left move to the front
        _case("compact_half", op="compact", seqs=256, ctx_lo=50, ctx_hi=2000, spare=0.5, layers=4),
    ]


def _log_int(rng, lo, hi):
    """Spread over the logarithm; whole thousands (of 1024) of tokens get one more."""
    n = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    return n + 1 if n > 1024 and n % 1024 == 0 and n < hi else n


_HEADS = ((32, 8, 128), (32, 8, 128), (16, 2, 128), (8, 1, 128), (14, 14, 64), (9, 3, 64), (20, 5, 80), (12, 2, 96), (8, 4, 256),
          (40, 8, 128), (7, 7, 40), (64, 8, 64))


def draw(rng):
    op = rng.choice(["append", "append", "attend", "attend", "attend", "attend", "attend", "pages", "pages", "compact"])
    shape = rng.randrange(1, 1 << 20)
    heads, kv, dim = rng.choice(_HEADS)
    common = dict(op=op, heads=heads, kv=kv, dim=dim, page=rng.choice([8, 16, 16, 32, 64]), slot_major=rng.random() < 0.3,
                  shape=shape)
    if op == "append":
        seqs = _log_int(rng, 1, 256)
        rot = rng.choice([dim, dim, dim // 2 // 8 * 8])
        lo = _log_int(rng, 1, 4000)
        return _case(seqs=seqs, rows=max(seqs, _log_int(rng, 1, 8000)), split=rng.choice(["even", "ragged"]), ctx_lo=lo,
                     ctx_hi=_log_int(rng, lo, max(lo + 1, min(120000, 1000000 // seqs))), rot=rot,
                     pairing=rng.choice(["half", "interleaved"]), scaling=rng.choice(["plain", "linear", "base", "parts"]),
                     f32=rng.random() < 0.3, fused=rng.random() < 0.6, **common)
    if op == "attend":
        kind = rng.choice(["decode", "decode", "verify", "prefill", "mixed", "cross"])
        lse = rng.random() < 0.3
        window = _log_int(rng, 16, 4000) if rng.random() < 0.25 else 0
        if kind in ("decode", "verify"):
            seqs = _log_int(rng, 1, 256)
            hi = _log_int(rng, 16, max(32, min(130000, 600000 // seqs)))
            rows = seqs if kind == "decode" else _log_int(rng, seqs, 8 * seqs)
            return _case(seqs=seqs, rows=rows, split="even" if kind == "decode" else "ragged", ctx_lo=max(1, hi // 30), ctx_hi=hi,
                         window=window, lse=lse, **common)
        if kind == "prefill":
            seqs = _log_int(rng, 1, 16)
            return _case(seqs=seqs, rows=max(seqs, min(_log_int(rng, 64, 16000), 1500 * seqs)), split=rng.choice(["even", "ragged"]),
                         ctx_lo=0, ctx_hi=_log_int(rng, 1, 500), window=window, lse=lse, **common)
        if kind == "mixed":
            seqs = _log_int(rng, 2, 64)
            lo = _log_int(rng, 10, 1000)
            return _case(seqs=seqs, rows=seqs + _log_int(rng, 64, 1900), split="mixed", ctx_lo=lo, ctx_hi=_log_int(rng, lo, 12000),
                         window=window, lse=lse, **common)
        # every row sees all that its sequence has cached, as over an encoder's states; some have none
        seqs = _log_int(rng, 1, 32)
        return _case(seqs=seqs, rows=_log_int(rng, seqs, 4000), split="ragged", ctx_lo=0, ctx_hi=_log_int(rng, 16, 3000),
                     causal=False, lse=lse, **common)
    seqs, lo = _log_int(rng, 2, 256), _log_int(rng, 1, 400)
    return _case(seqs=seqs, ctx_lo=lo, ctx_hi=_log_int(rng, lo, max(lo + 1, min(4000, 130000 // seqs))), layers=rng.choice([1, 2, 3, 4]),
                 width=rng.choice([1, 2, 4, 8]), done=rng.choice([0.0, 0.1, 0.3]), spare=rng.choice([0.2, 0.4, 0.5]), **common)


def _lengths(case):
    """(new rows, length with them) of every sequence, which the case alone decides."""
    rng = np.random.RandomState(case["shape"])
    n, total = case["seqs"], case["rows"]
    lo, hi = case["ctx_lo"], case["ctx_hi"]
    ctx = np.rint(np.exp(rng.uniform(math.log(lo + 1), math.log(hi + 1), n)) - 1).astype(np.int64)
    if case["op"] in ("pages", "compact"):
        return np.zeros(n, np.int64), np.maximum(ctx, 1)
    if case["split"] == "even":
        rows = np.full(n, total // n) + (np.arange(n) < total % n)
    elif case["split"] == "mixed":
        rows = np.ones(n, np.int64)
        rows[rng.randint(n)] = total - n + 1
        ctx[rows > 1] = hi
    else:
        rows = rng.multinomial(total, rng.dirichlet(np.full(n, 1.5)))
    return rows.astype(np.int64), (rows + ctx if case["causal"] else ctx).astype(np.int64)


def _pages_of(tokens, page):
    return -(-tokens // page)


def _plan_of(case):
    """pages: which slot every slot's tokens come from, and its new length, as the server decided."""
    rng = np.random.RandomState(case["shape"] + 1)
    n, width = case["seqs"], case["width"]
    _, lens = _lengths(case)
    parents = _pages_of(n, width) if width > 1 else n
    lens[parents:] = 0
    src = np.arange(n)
    if width > 1:                       # slot i < parents is a prompt; the slots behind take it over in turn
        src = np.arange(n) % parents
    new = lens[src] + 1
    gone = rng.rand(n) < case["done"]
    new[gone] = np.where(rng.rand(n) < 0.5, 0, lens[src] // 2)[gone]
    if width == 1 and n >= 8:           # a finished sequence's slot goes to a copy of another one
        for s in np.nonzero(gone)[0][:2]:
            src[s] = (s + 1) % n
            new[s] = lens[src[s]] + 1
    return lens, src.astype(np.int64), new.astype(np.int64)


_SCALING = dict(plain=0, linear=1, base=2, parts=3)


def _rope_args(case):
    long = case["scaling"] != "plain"
    return dict(rot_dim=case["rot"], base=500000.0 if case["scaling"] == "parts" else 10000.0, scaling=_SCALING[case["scaling"]],
                factor=8.0 if long else 1.0, original_len=8192.0, low=1.0, high=4.0,
                amplitude=0.1 * math.log(8.0) + 1.0 if case["scaling"] == "parts" else 1.0)


def _frequencies(case):
    """Radians per position of every rotated pair, in 64 bits."""
    a = _rope_args(case)
    i = np.arange(a["rot_dim"] // 2, dtype=np.float64)
    base = a["base"]
    if case["scaling"] == "base" and a["rot_dim"] > 2:
        base *= a["factor"] ** (a["rot_dim"] / (a["rot_dim"] - 2.0))
    f = base ** (-2.0 * i / a["rot_dim"])
    if case["scaling"] == "linear":
        f = f / a["factor"]
    if case["scaling"] == "parts":
        turns = a["original_len"] * f / (2 * math.pi)
        part = np.clip((turns - a["low"]) / (a["high"] - a["low"]), 0.0, 1.0)
        f = (1 - part) * f / a["factor"] + part * f
    return f


def _cache(case, pages, gen):
    """K and V as [layer][page][head][token][width], whatever the order in memory."""
    L, P, H, S, D = case["layers"], pages, case["kv"], case["page"], case["dim"]
    both = []
    for _ in range(2):
        t = torch.randn((L, P, S, H, D) if case["slot_major"] else (L, P, H, S, D), generator=gen, device="cuda", dtype=torch.bfloat16)
        both.append(t.transpose(2, 3) if case["slot_major"] else t)
    return both


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    host = np.random.RandomState(seed)
    H, KV, D, page = case["heads"], case["kv"], case["dim"], case["page"]
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()     # noqa: E731
    st = dict(case=case)
    if case["op"] in ("pages", "compact"):
        if case["op"] == "pages":
            lens, src, new = _plan_of(case)
            wanted = int((_pages_of(new, page) - _pages_of(np.minimum(lens[src], new), page)).sum()) + len(new)
        else:
            lens, src, new, wanted = _lengths(case)[1], None, None, 0
    else:
        rows, lens = _lengths(case)
    held = _pages_of(lens, page)
    used = int(held.sum())
    if case["op"] == "pages":
        used = max(used, 1) + wanted
    n_pages = max(4, int(math.ceil(used / (1.0 - case["spare"]))))
    order = host.permutation(n_pages)
    most = int(max(1, held.max(), _pages_of(new, page).max() if case["op"] == "pages" else 0))
    table = np.full((len(lens), most), -1, np.int32)
    at = 0
    for s, h in enumerate(held):
        table[s, :h] = order[at:at + h]
        at += h
    st["table"], st["len"] = dev(table), dev(lens)
    st["k"], st["v"] = _cache(case, n_pages, gen)
    if case["op"] in ("pages", "compact"):
        st["to"] = dict(table=torch.empty_like(st["table"]), len=torch.empty_like(st["len"]),
                        ref=torch.empty(n_pages, dtype=torch.int32, device="cuda"))
        if src is not None:
            st["src"], st["new"] = dev(src), dev(new)
    else:
        T = int(rows.sum())
        st["start"] = dev(np.concatenate([[0], np.cumsum(rows)]))
        st["rows"], st["lens"] = rows, lens        # what a scheduler knows on the host
        if case["op"] == "append":
            kind = torch.float32 if case["f32"] else torch.bfloat16
            if case["fused"]:
                x = torch.randn((T, (H + 2 * KV) * D), generator=gen, device="cuda").to(kind)
                st["q"], st["nk"], st["nv"] = x[:, :H * D], x[:, H * D:(H + KV) * D], x[:, (H + KV) * D:]
            else:
                st["q"], st["nk"], st["nv"] = (torch.randn((T, h * D), generator=gen, device="cuda").to(kind) for h in (H, KV, KV))
            st["q_out"] = torch.empty((T, H * D), dtype=torch.bfloat16, device="cuda")
            st["freq"] = torch.from_numpy(_frequencies(case)).cuda()
        else:
            st["q"] = (1.7 * torch.randn((T, H * D), generator=gen, device="cuda")).to(torch.bfloat16)
            st["out"] = torch.empty_like(st["q"])
            st["lse"] = torch.empty((T, H), dtype=torch.float32, device="cuda") if case["lse"] else None
    if own:                                        # the handles that a user's program keeps
        import paper_2604_07173_amd as L
        st["cache"] = L.KvCache(st["k"], st["v"])
        if case["op"] in ("pages", "compact"):
            t = st["to"]
            st["from_c"] = L.KvState(st["table"], st["len"])
            st["to_c"] = L.KvState(t["table"], t["len"], page_ref=t["ref"])
            st["moves"] = L.KvMoves(n_pages, len(lens))
        else:
            st["batch"] = L.KvBatch(st["start"], st["len"], st["table"], n_rows=T, max_rows=int(rows.max()))
            if case["op"] == "append":
                st["rope"] = L.Rope(pairing=L.LORA_ROPE_HALF if case["pairing"] == "half" else L.LORA_ROPE_INTERLEAVED,
                                    **_rope_args(case))
            else:
                st["ws"] = torch.empty(max(256, L.lora_kv_attention_ws_bytes(st["cache"], st["batch"], H)), dtype=torch.uint8,
                                       device="cuda")
    return st


def run(st):
    case = st["case"]
    return {"append": _append, "attend": _attend, "pages": _pages, "compact": _compact}[case["op"]](st, case)


# ---- rotary positions and the append -------------------------------------------------------------------


def _row_places(st):
    """Sequence of every new row and its position there."""
    T = st["q"].shape[0]
    t = torch.arange(T, device="cuda", dtype=torch.int32)
    seq = torch.searchsorted(st["start"], t, right=True) - 1
    return seq, st["len"][seq].long() - st["start"][seq + 1].long() + t.long()


def _rotated(x, heads, dim, angle, amplitude, rot, pairing):
    x = x.float().view(x.shape[0], heads, dim)
    cos, sin = (angle.cos() * amplitude).float()[:, None, :], (angle.sin() * amplitude).float()[:, None, :]
    head = x[..., :rot]
    a, b = (head[..., :rot // 2], head[..., rot // 2:]) if pairing == "half" else (head[..., 0::2], head[..., 1::2])
    first, second = a * cos - b * sin, a * sin + b * cos
    turned = torch.cat([first, second], -1) if pairing == "half" else torch.stack([first, second], -1).flatten(-2)
    return torch.cat([turned, x[..., rot:]], -1)


def _append(st, case):
    H, KV, D = case["heads"], case["kv"], case["dim"]
    if own:
        import paper_2604_07173_amd as L
        L.lora_rope_append(st["cache"], 0, st["batch"], st["rope"], st["q"], st["q"].stride(0), st["nk"], st["nk"].stride(0),
                           st["nv"], st["nv"].stride(0), st["q_out"], H * D, H,
                           L.LORA_DTYPE_F32 if case["f32"] else L.LORA_DTYPE_BF16)
        return st["q_out"], st["k"], st["v"]
    seq, pos = _row_places(st)
    angle = pos.double()[:, None] * st["freq"]       # the position times a frequency that came in 64 bits
    amplitude = _rope_args(case)["amplitude"]
    T = pos.shape[0]
    st["q_out"].copy_(_rotated(st["q"], H, D, angle, amplitude, case["rot"], case["pairing"]).view(T, H * D))
    page = st["table"][seq, pos // case["page"]].long()
    slot = pos % case["page"]
    st["k"][0].transpose(1, 2)[page, slot] = _rotated(st["nk"], KV, D, angle, amplitude, case["rot"], case["pairing"]).bfloat16()
    st["v"][0].transpose(1, 2)[page, slot] = st["nv"].bfloat16().view(T, KV, D)
    return st["q_out"], st["k"], st["v"]


# ---- attention -----------------------------------------------------------------------------------------


def _seen(case, n_rows, length, pos0, tokens):
    """[..][row][token]: what a row may look at."""
    j = torch.arange(tokens, device="cuda")
    pos = pos0[..., None, None] + torch.arange(n_rows, device="cuda")[:, None]
    seen = j < length[..., None, None]
    if case["causal"]:
        seen = seen & (j <= pos)
        if case["window"]:
            seen = seen & (j > pos - case["window"])
    return seen.expand(*seen.shape[:-2], n_rows, tokens)


def _attend_padded(st, case, q, table, length, pos0):
    """q [n][r][heads][dim] over the tables' pages, all sequences padded to the tables' width."""
    n, r = q.shape[:2]
    KV, D, G = case["kv"], case["dim"], case["heads"] // case["kv"]
    tokens = table.shape[1] * case["page"]
    k = st["k"][0][table.clamp(min=0)].transpose(1, 2).reshape(n, KV, tokens, D)
    v = st["v"][0][table.clamp(min=0)].transpose(1, 2).reshape(n, KV, tokens, D)
    q = q.float().view(n, r, KV, G, D).transpose(1, 2).reshape(n, KV, r * G, D)
    s = torch.matmul(q * (1.0 / math.sqrt(D)), k.float().transpose(2, 3).contiguous()).view(n, KV, r, G, tokens)
    seen = _seen(case, r, length, pos0, tokens)
    s = s.masked_fill(~seen[:, None, :, None, :], -math.inf)
    top = s.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, torch.zeros_like(top), top)
    p = (s - top).exp()
    total = p.sum(-1, keepdim=True)
    live = torch.arange(tokens, device="cuda") < length[:, None]
    v = torch.where(live[:, None, :, None], v.float(), torch.zeros((), device="cuda"))
    o = torch.matmul(p.view(n, KV, r * G, tokens), v).view(n, KV, r, G, D)
    o = o / torch.where(total == 0, torch.ones_like(total), total)
    lse = (top + total.log()).squeeze(-1)
    heads = KV * G
    return o.transpose(1, 2).reshape(n, r, heads * D), lse.transpose(1, 2).reshape(n, r, heads)


def _attend(st, case):
    H, D = case["heads"], case["dim"]
    if own:
        import paper_2604_07173_amd as L
        L.lora_kv_attention(st["cache"], 0, st["batch"], st["q"], H * D, H, st["out"], H * D, st["lse"], 1.0 / math.sqrt(D),
                            st["ws"], causal=case["causal"], window=case["window"])
        return (st["out"], st["lse"]) if case["lse"] else (st["out"],)
    rows, lens, page = st["rows"], st["lens"], case["page"]
    starts = np.concatenate([[0], np.cumsum(rows)])
    few = int(rows.max()) if rows.max() <= 32 else 1
    lse = torch.empty((st["q"].shape[0], H), device="cuda")
    short = [s for s in range(len(rows)) if 0 < rows[s] <= few]
    if short:                                       # all of them at once, padded to `few` rows
        first = torch.tensor([int(starts[s]) for s in short], device="cuda")
        count = torch.tensor([int(rows[s]) for s in short], device="cuda")
        which = torch.tensor(short, device="cuda")
        i = torch.arange(few, device="cuda")
        at = first[:, None] + torch.minimum(i, count[:, None] - 1)
        table = st["table"][which, :max(1, _pages_of(max(int(lens[s]) for s in short), page))].long()
        length = st["len"][which].long()
        o, e = _attend_padded(st, case, st["q"][at].view(len(short), few, H, D), table, length, length - count)
        mine = (i < count[:, None]).flatten()
        st["out"][at.flatten()[mine]] = o.flatten(0, 1)[mine].bfloat16()
        lse[at.flatten()[mine]] = e.flatten(0, 1)[mine]
    for s in np.nonzero(rows > few)[0]:             # a long chunk by itself
        a, b = int(starts[s]), int(starts[s + 1])
        table = st["table"][s:s + 1, :max(1, _pages_of(int(lens[s]), page))].long()
        length = st["len"][s:s + 1].long()
        o, e = _attend_padded(st, case, st["q"][a:b].view(1, b - a, H, D), table, length, length - (b - a))
        st["out"][a:b] = o[0].bfloat16()
        lse[a:b] = e[0]
    if case["lse"]:
        st["lse"].copy_(lse)
        return st["out"], st["lse"]
    return (st["out"],)


# ---- pages ---------------------------------------------------------------------------------------------


def _copy_pages(st, src, dst):
    for t in (st["k"], st["v"]):
        t[:, dst] = t[:, src]


def _result(st, table, length, ref, copies, wanted):
    to, n_pages = st["to"], ref.shape[0]
    to["table"].copy_(table)
    to["len"].copy_(length)
    to["ref"].copy_(ref)
    used = (ref > 0).sum()
    return dict(to, counts=torch.stack([used, copies, n_pages - used, wanted]).int(), k=st["k"], v=st["v"])


def _ranked(flags, ids, room):
    """ids[flags], in order, in a list of fixed length (the rest -1), without a count on the host."""
    place = torch.where(flags, flags.long().cumsum(0) - 1, room)
    return torch.full((room + 1,), -1, dtype=torch.long, device="cuda").scatter_(0, place, ids)[:room]


def _pages(st, case):
    page, n_pages = case["page"], st["k"].shape[1]
    if own:
        import paper_2604_07173_amd as L
        L.lora_kv_plan(st["cache"], st["from_c"], st["to_c"], st["src"], st["new"], st["moves"])
        L.lora_kv_copy_pages(st["cache"], st["moves"], max_moves=len(st["new"]))
        return dict(st["to"], counts=st["moves"].counts, k=st["k"], v=st["v"])
    src, new = st["src"].long(), st["new"].long()
    n, most = st["table"].shape
    slots, col = torch.arange(n, device="cuda"), torch.arange(most, device="cuda")
    keep = torch.minimum(torch.where(src >= 0, st["len"].long()[src.clamp(min=0)], 0), new)
    kp, np_ = -(-keep // page), -(-new // page)
    rows = st["table"].long()[src.clamp(min=0)]
    kept = col < kp[:, None]
    spill = torch.where(kept, rows, n_pages).flatten()          # one place past the pages takes what does not count
    ref = torch.zeros(n_pages + 1, dtype=torch.long, device="cuda").scatter_add_(0, spill, torch.ones_like(spill))
    ref[n_pages] = 0
    grows = (new > keep) & (keep % page != 0)
    last = torch.where(grows, rows.gather(1, (kp - 1).clamp(min=0)[:, None])[:, 0], n_pages)
    growing = torch.zeros_like(ref).scatter_add_(0, last, torch.ones_like(last))
    lowest = torch.full_like(ref, n).scatter_reduce_(0, last, slots, "amin")
    keeps = (growing[last] == ref[last]) & (lowest[last] == slots)
    cow = grows & (ref[last] > 1) & ~keeps
    need = cow.long() + np_ - kp
    base = need.cumsum(0) - need
    pages = torch.arange(n_pages, device="cuda")
    free = _ranked(ref[:n_pages] == 0, pages, n_pages)
    grown = (base + cow.long())[:, None] + col - kp[:, None]
    table = torch.where(kept, rows, torch.where(col < np_[:, None], free[grown.clamp(0, n_pages - 1)], -1))
    own_page = free[base.clamp(max=n_pages - 1)]
    table = torch.where(cow[:, None] & (col == kp[:, None] - 1), own_page[:, None], table)
    spill = torch.where(col < np_[:, None], table, n_pages).flatten()
    after = torch.zeros(n_pages + 1, dtype=torch.long, device="cuda").scatter_add_(0, spill, torch.ones_like(spill))[:n_pages]
    still = (ref[:n_pages] > 0).long().argmax()                 # a page that nobody writes, for the slots without a copy
    _copy_pages(st, torch.where(cow, last, still), torch.where(cow, own_page, still))
    return _result(st, table, new, after, cow.sum(), need.sum())


def _compact(st, case):
    n_pages = st["k"].shape[1]
    if own:
        import paper_2604_07173_amd as L
        L.lora_kv_compact(st["cache"], st["from_c"], st["to_c"], st["moves"])
        L.lora_kv_copy_pages(st["cache"], st["moves"], max_moves=n_pages // 2)
        return dict(st["to"], counts=st["moves"].counts, k=st["k"], v=st["v"])
    n, most = st["table"].shape
    col = torch.arange(most, device="cuda")
    held = col < (-(-st["len"].long() // case["page"]))[:, None]
    table = torch.where(held, st["table"].long(), n_pages)
    ref = torch.zeros(n_pages + 1, dtype=torch.long, device="cuda").scatter_add_(0, table.flatten(), torch.ones_like(table.flatten()))
    live = ref[:n_pages] > 0
    pages = torch.arange(n_pages, device="cuda")
    n_live = live.sum()
    mover, hole = live & (pages >= n_live), ~live & (pages < n_live)
    half = n_pages // 2
    src, dst = _ranked(mover, pages, half), _ranked(hole, pages, half)
    to = torch.where(mover, dst[(mover.long().cumsum(0) - 1).clamp(0, half - 1)], pages)
    still = n_pages - 1                                         # never a hole's number
    _copy_pages(st, torch.where(src >= 0, src, still), torch.where(src >= 0, dst, still))
    moved = torch.cat([to, torch.full((1,), -1, device="cuda")])[table]
    after = torch.zeros_like(ref).scatter_add_(0, torch.where(held, moved, n_pages).flatten(), torch.ones_like(moved.flatten()))
    return _result(st, moved, st["len"], after[:n_pages], mover.sum(), torch.zeros_like(n_live))


# ---- what a pass cannot do without, and the exact results ----------------------------------------------


def work(case):
    H, KV, D, page = case["heads"], case["kv"], case["dim"], case["page"]
    if case["op"] == "append":
        T = case["rows"]
        each = 4 if case["f32"] else 2
        return dict(bytes=T * (H + 2 * KV) * D * (each + 2), flops=T * (H + KV) * case["rot"] * 3)
    if case["op"] == "attend":
        rows, lens = _lengths(case)
        pairs, tokens = 0, 0
        for r, n in zip(rows, lens):
            if r == 0:
                continue
            if not case["causal"]:
                pairs, tokens = pairs + int(r * n), tokens + int(n)
                continue
            w = case["window"] or int(n)
            last = np.arange(n - r + 1, n + 1)
            pairs += int(np.minimum(last, w).sum())
            tokens += int(min(n, w + r - 1))
        T = int(rows.sum())
        return dict(bytes=tokens * KV * D * 4 + T * H * D * 4 + (T * H * 4 if case["lse"] else 0), flops=pairs * H * D * 4)
    if case["op"] == "pages":
        lens, src, new = _plan_of(case)
        # every slot that writes into the middle of a page that another one keeps needs one of its own
        keep = np.minimum(lens[src], new)
        kp = _pages_of(keep, page)
        holders = {}
        for s in np.nonzero(kp)[0]:
            for c in range(int(kp[s])):
                holders.setdefault((int(src[s]), c), []).append(s)
        copies = 0
        for s in np.nonzero((new > keep) & (keep % page != 0))[0]:
            same = holders[(int(src[s]), int(kp[s]) - 1)]
            writers = [u for u in same if new[u] > keep[u] and keep[u] % page and kp[u] == kp[s]]
            copies += len(same) > 1 and not (len(writers) == len(same) and min(writers) == s)
        entries = int(kp.sum()) + int(_pages_of(new, page).sum())
    else:
        lens = _lengths(case)[1]
        live = int(_pages_of(lens, page).sum())
        n_pages = max(4, int(math.ceil(live / (1.0 - case["spare"]))))
        copies, entries = int(live * (1 - live / n_pages)), 2 * live     # the pages behind the first `live`, on average
    moved = copies * case["layers"] * page * KV * D * 2 * 2
    return dict(bytes=2 * moved + 4 * entries, flops=entries)


def exact(case, seed):
    if case["op"] in ("pages", "compact"):
        return None                                  # page numbers and copies: nothing is computed in floating point
    global own
    mine, own = own, False
    try:
        st = prepare(case, seed)
    finally:
        own = mine
    rows, lens = _lengths(case)
    H, KV, D, page = case["heads"], case["kv"], case["dim"], case["page"]
    table = st["table"].cpu().numpy()
    starts = np.concatenate([[0], np.cumsum(rows)])
    if case["op"] == "append":
        q = st["q"].double().view(-1, H, D).clone()
        nk, nv = st["nk"].double().view(-1, KV, D).clone(), st["nv"].double().view(-1, KV, D)
        k, v = st["k"].double(), st["v"].double()
        pos = np.concatenate([np.arange(n - r, n) for r, n in zip(rows, lens)])
        turn = np.exp(1j * pos[:, None] * _frequencies(case)[None, :]) * _rope_args(case)["amplitude"]
        turn = torch.from_numpy(turn).cuda()[:, None, :]
        rot = case["rot"]
        even = torch.arange(0, rot // 2, device="cuda") if case["pairing"] == "half" else torch.arange(0, rot, 2, device="cuda")
        odd = even + (rot // 2 if case["pairing"] == "half" else 1)
        for x in (q, nk):                            # a pair as a complex number, turned by its angle
            z = torch.complex(x[..., even], x[..., odd]) * turn
            x[..., even], x[..., odd] = z.real, z.imag
        pages = np.concatenate([table[s, np.arange(lens[s] - r, lens[s]) // page] for s, r in enumerate(rows)])
        to = torch.from_numpy(pages.astype(np.int64)).cuda() * page + torch.from_numpy(pos % page).cuda()
        for cache, x in ((k, nk), (v, nv)):
            flat = cache[0].permute(0, 2, 1, 3).reshape(-1, KV, D).clone()
            flat[to] = x
            cache[0] = flat.view(cache.shape[1], page, KV, D).permute(0, 2, 1, 3)
        return q.view(-1, H * D), k, v
    G = H // KV
    out = torch.zeros((int(rows.sum()), H, D), dtype=torch.float64, device="cuda")
    lse = torch.full((int(rows.sum()), H), -math.inf, dtype=torch.float64, device="cuda")
    for s, (r, n) in enumerate(zip(rows, lens)):
        if r == 0 or n == 0:
            continue
        pages = torch.from_numpy(table[s, :_pages_of(n, page)].astype(np.int64)).cuda()
        for h in range(KV):
            k = st["k"][0, pages, h].reshape(-1, D)[:n].double()
            v = st["v"][0, pages, h].reshape(-1, D)[:n].double()
            for a in range(0, r, 2048):
                b = min(r, a + 2048)
                at = slice(int(starts[s]) + a, int(starts[s]) + b)
                q = st["q"][at].view(-1, H, D)[:, h * G:(h + 1) * G].double().reshape(-1, D)
                score = (q @ k.t() / math.sqrt(D)).view(b - a, G, n)
                if case["causal"]:
                    where = torch.arange(n - r + a, n - r + b, device="cuda")[:, None]
                    token = torch.arange(n, device="cuda")[None, :]
                    hidden = token > where
                    if case["window"]:
                        hidden = hidden | (token <= where - case["window"])
                    score = score.masked_fill(hidden[:, None, :], -math.inf)
                lse[at, h * G:(h + 1) * G] = torch.logsumexp(score, -1)
                out[at, h * G:(h + 1) * G] = (torch.softmax(score, -1).view(-1, n) @ v).view(b - a, G, D)
    out = out.view(-1, H * D)
    return (out, lse) if case["lse"] else (out,)
