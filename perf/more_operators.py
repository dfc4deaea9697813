"""Timed cases of a decode step in which several answers to one prompt are drawn: the search for sequences that hold the same
first pages, attention that reads such pages once for all of them, the residual's addition with the norm behind it, and
the choice of the next tokens.

A case is one call.  `own` says who computes it: False the plain form of this file, in torch operations of 32 bits
(64 where sums are long or decide between tokens) that are rounded once at the end, True the library's entry points.

Fields of a case:
  op          "share", "attend", "norm" or "sample"
  share, attend:
  seqs        sequences of the batch;  prompts: how many prompts they answer;  split: "even" or "ragged" (some prompts have one
              answer or none)
  prompt_lo, prompt_hi   tokens of a prompt, spread over the logarithm;  own_lo, own_hi: tokens of an answer so far
  most        new rows of a sequence: 1, or 0 to `most` of them (drafted tokens; some sequences pause)
  heads, kv, dim   query heads, key/value heads, width of a head
  page        tokens of a page;  slot_major: pages laid out [token][head] instead of [head][token]
  causal      attend: the mask;  lse: the logarithm of the softmax sum is asked for too
  shape       seed of the lengths, which belong to the case and not to its inputs
  norm:
  rows, width;  f32: the residual stream is held in 32 bits instead of bf16;  add: "none", "bf16" or "f32"
  y           the bf16 rows are asked for;  eight: columns that share a scale of the 8-bit rows (0: the whole row, -1: none asked for)
  shift       added to the weights (1: weights are held as differences from one)
  sample:
  rows, vocab;  f32: logits in 32 bits instead of bf16;  pad: unused columns behind the vocabulary
  rule        "topk_topp", "topp", "minp", "plain" (temperature only), "greedy" or "mixed" (every row has its own)
"""
import math

import numpy as np
import torch

own = False

_DEFAULTS = dict(
    attend=dict(op="attend", seqs=1, prompts=1, split="even", prompt_lo=16, prompt_hi=16, own_lo=0, own_hi=0, most=1, heads=32, kv=8,
                dim=128, page=16, slot_major=False, causal=True, lse=False, shape=1),
    norm=dict(op="norm", rows=1, width=4096, f32=False, add="bf16", y=True, eight=-1, shift=0.0),
    sample=dict(op="sample", rows=1, vocab=32000, f32=True, pad=0, rule="topk_topp"))
_DEFAULTS["share"] = dict(_DEFAULTS["attend"], op="share")

_MAX_ROWS = 16             # a sequence with more new rows gains nothing from sharing: it fills a tile by itself
_EPS = 1e-5
_E4M3_MOST = 448.0


def _case(name=None, **kw):
    base = _DEFAULTS[kw["op"]]
    unknown = set(kw) - set(base)
    if unknown:
        raise ValueError(f"unknown fields {sorted(unknown)}")
    c = dict(base, **kw)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # one step of a small server: four prompts with sixteen answers each
        _case("share_64", op="share", seqs=64, prompts=4, prompt_lo=1000, prompt_hi=3000, own_lo=1, own_hi=400),
        # a full server: 1024 slots, prompts of all lengths with one to many answers
        _case("share_1024", op="share", seqs=1024, prompts=150, split="ragged", prompt_lo=100, prompt_hi=12000, own_lo=0, own_hi=800, most=3),
        # eight answers to one prompt: latency
        _case("attend_shared_8", op="attend", seqs=8, prompts=1, prompt_lo=1500, prompt_hi=1500, own_lo=1, own_hi=40),
        # sixteen answers to each of sixteen prompts
        _case("attend_shared_256", op="attend", seqs=256, prompts=16, prompt_lo=1000, prompt_hi=6000, own_lo=20, own_hi=1000),
        # many answers over one long document
        _case("attend_shared_long", op="attend", seqs=128, prompts=1, prompt_lo=32000, prompt_hi=32000, own_lo=10, own_hi=500, lse=True),
        # drafted tokens of uneven groups are verified, odd heads, prompts that end inside a page
        _case("attend_shared_verify", op="attend", seqs=61, prompts=9, split="ragged", prompt_lo=50, prompt_hi=5000, own_lo=0, own_hi=300,
              most=6, heads=20, kv=5, dim=80, page=8, slot_major=True),
        # a decode batch's residual and norm in front of the q, k and v products
        _case("norm_decode_64", op="norm", rows=64),
        # an odd batch over a residual stream in 32 bits, 8-bit rows with one scale each beside the bf16 ones
        _case("norm_odd_f32", op="norm", rows=1333, width=2056, f32=True, add="f32", eight=0, shift=1.0),
        # the prefill workload's rows, for a base product in 8 bits with scales for every 128 columns
        _case("norm_prefill_16384", op="norm", rows=16384, eight=128),
        # one user's next token
        _case("sample_1", op="sample", rows=1, vocab=32000),
        # a batch whose users have settings of their own, a large vocabulary
        _case("sample_64", op="sample", rows=64, vocab=128000, rule="mixed"),
        # many answers at once, an odd vocabulary in bf16, where many logits are equal
        _case("sample_512_bf16", op="sample", rows=512, vocab=50257, f32=False, rule="topp"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


_HEADS = ((32, 8, 128), (32, 8, 128), (16, 2, 128), (8, 1, 128), (14, 14, 64), (9, 3, 64), (20, 5, 80), (12, 2, 96), (8, 4, 256),
          (40, 8, 128), (7, 7, 40), (64, 8, 64))


def draw(rng):
    op = rng.choice(["share", "attend", "attend", "attend", "norm", "norm", "sample", "sample"])
    if op in ("share", "attend"):
        heads, kv, dim = rng.choice(_HEADS)
        seqs = _log_int(rng, 16, 1024) if op == "share" else _log_int(rng, 2, 256)
        hi = _log_int(rng, 20, min(30000, 4000000 // seqs // 2))
        own_hi = _log_int(rng, 1, max(2, min(2000, 400000 // seqs)))
        return _case(op=op, seqs=seqs, prompts=_log_int(rng, 1, max(2, seqs // 2)), split=rng.choice(["even", "ragged"]),
                     prompt_lo=max(1, hi // rng.choice([1, 4, 30])), prompt_hi=hi, own_lo=rng.choice([0, 1, max(1, own_hi // 20)]),
                     own_hi=own_hi, most=rng.choice([1, 1, 2, 5, 8]), heads=heads, kv=kv, dim=dim, page=rng.choice([8, 16, 16, 32, 64]),
                     slot_major=rng.random() < 0.3, causal=rng.random() < 0.9, lse=rng.random() < 0.3, shape=rng.randrange(1, 1 << 20))
    if op == "norm":
        width = 8 * _log_int(rng, 8, 2048)
        return _case(op=op, rows=_log_int(rng, 1, min(20000, 60000000 // width)), width=width, f32=rng.random() < 0.3,
                     add=rng.choice(["none", "bf16", "bf16", "f32"]), eight=rng.choice([-1, -1, 0, 32, 128]),
                     shift=rng.choice([0.0, 0.0, 1.0]))
    vocab = _log_int(rng, 100, 200000)
    return _case(op=op, rows=_log_int(rng, 1, min(1024, 26000000 // vocab)), vocab=vocab, f32=rng.random() < 0.6,
                 pad=rng.choice([0, 0, 1, 64]), rule=rng.choice(["topk_topp", "topp", "minp", "plain", "greedy", "mixed", "mixed"]))


# ---- sequences and their pages -------------------------------------------------------------------------


def _lengths(case):
    """(prompt of every sequence, its tokens, new rows, length with them), which the case alone decides."""
    rng = np.random.RandomState(case["shape"])
    n, prompts = case["seqs"], case["prompts"]
    spread = lambda lo, hi, k: np.rint(np.exp(rng.uniform(math.log(lo + 1), math.log(hi + 1), k)) - 1).astype(np.int64)     # noqa: E731
    of = np.arange(n) % prompts if case["split"] == "even" else rng.randint(0, prompts, n)
    prompt = spread(case["prompt_lo"], case["prompt_hi"], prompts)[of]
    mine = spread(case["own_lo"], case["own_hi"], n)
    rows = np.ones(n, np.int64)
    if case["most"] > 1:
        rows = rng.randint(0, case["most"] + 1, n)
        rows[rng.randint(n)] = case["most"]
    if case["op"] == "share":
        rows[3::7] = 0                               # some sequences pause
    return of, prompt, rows, prompt + mine + rows


def _tables(case, host):
    """Pages of every sequence: the prompt's whole pages are those of all its answers.  Returns the tables and the number of pages."""
    of, prompt, _, lens = _lengths(case)
    page = case["page"]
    held, whole = -(-lens // page), prompt // page
    taken = np.zeros(case["prompts"], np.int64)
    taken[of] = whole
    n_pages = int(taken.sum() + (held - whole).sum()) + 5
    order = host.permutation(n_pages)
    first, more = np.cumsum(taken) - taken, held - whole
    at = int(taken.sum()) + np.cumsum(more) - more
    col = np.arange(int(held.max()))
    place = np.where(col < whole[:, None], first[of][:, None] + col, (at - whole)[:, None] + col)
    return np.where(col < held[:, None], order[np.minimum(place, n_pages - 1)], -1).astype(np.int32), n_pages


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    host = np.random.RandomState(seed)
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()                     # noqa: E731
    st = dict(case=case)
    if case["op"] in ("share", "attend"):
        H, KV, D, page = case["heads"], case["kv"], case["dim"], case["page"]
        _, _, rows, lens = _lengths(case)
        table, n_pages = _tables(case, host)
        T = int(rows.sum())
        if case["op"] == "share":                  # which slot holds which sequence
            order = host.permutation(case["seqs"])
            table, rows, lens = table[order], rows[order], lens[order]
        st["table"], st["len"] = dev(table), dev(lens.astype(np.int32))
        st["start"] = dev(np.concatenate([[0], np.cumsum(rows)]).astype(np.int32))
        st["most"], st["n_rows"] = int(rows.max()), T
        if case["op"] == "attend":
            shape = (1, n_pages, page, KV, D) if case["slot_major"] else (1, n_pages, KV, page, D)
            st["k"], st["v"] = (torch.randn(shape, generator=gen, device="cuda", dtype=torch.bfloat16) for _ in range(2))
            if case["slot_major"]:
                st["k"], st["v"] = st["k"].transpose(2, 3), st["v"].transpose(2, 3)
            st["q"] = (1.7 * torch.randn((T, H * D), generator=gen, device="cuda")).to(torch.bfloat16)
            st["out"] = torch.empty_like(st["q"])
            st["lse"] = torch.empty((T, H), dtype=torch.float32, device="cuda") if case["lse"] else None
        else:
            # the search looks at tables only: a cache of one narrow head
            st["k"], st["v"] = (torch.zeros((1, n_pages, 1, page, 8), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    elif case["op"] == "norm":
        R, W = case["rows"], case["width"]
        make = lambda kind, scale: (scale * torch.randn((R, W), generator=gen, device="cuda")).to(kind)        # noqa: E731
        st["x"] = make(torch.float32 if case["f32"] else torch.bfloat16, 3.0)
        st["add"] = None if case["add"] == "none" else make(torch.float32 if case["add"] == "f32" else torch.bfloat16, 1.0)
        st["weight"] = (1.0 - case["shift"] + 0.2 * torch.randn(W, generator=gen, device="cuda")).to(torch.bfloat16)
        st["sum"] = torch.empty_like(st["x"])
        st["y"] = torch.empty((R, W), dtype=torch.bfloat16, device="cuda") if case["y"] else None
        if case["eight"] >= 0:
            groups = -(-W // case["eight"]) if case["eight"] else 1
            st["y8"] = torch.empty((R, W), dtype=torch.float8_e4m3fn, device="cuda")
            st["scale"] = torch.empty((R, groups), dtype=torch.float32, device="cuda")
    else:
        R, V = case["rows"], case["vocab"]
        x = 2.2 * torch.randn((R, V + case["pad"]), generator=gen, device="cuda")
        # a few likely tokens stand out, in some rows more than in others
        likely = torch.randint(0, V, (R, 24), generator=gen, device="cuda")
        lift = 12.0 * torch.rand((R, 24), generator=gen, device="cuda") * torch.rand((R, 1), generator=gen, device="cuda")
        x.scatter_add_(1, likely, lift)
        st["logits"] = x if case["f32"] else x.to(torch.bfloat16)
        one = np.ones(R, np.float32)
        pick = lambda *v: np.array(v)[host.randint(0, len(v), R)]                        # noqa: E731
        rule = {
            "topk_topp": lambda: (0.8 * one, 50 * one, 0.9 * one, 0 * one),
            "topp": lambda: (one, 0 * one, 0.95 * one, 0 * one),
            "minp": lambda: (1.3 * one, 0 * one, one, 0.05 * one),
            "plain": lambda: (0.9 * one, 0 * one, one, 0 * one),
            "greedy": lambda: (0 * one, 0 * one, one, 0 * one),
            "mixed": lambda: (pick(0.0, 0.3, 0.7, 1.0, 1.5), pick(0, 0, 1, 20, 400, 5000), pick(0.3, 0.9, 0.95, 0.99, 1.0), pick(0.0, 0.0, 0.02, 0.2)),
        }[case["rule"]]()
        st["temperature"], st["top_k"], st["top_p"], st["min_p"] = (dev(a.astype(t)) for a, t in zip(rule, (np.float32, np.int32, np.float32, np.float32)))
        st["u"] = torch.rand(R, generator=gen, device="cuda")
        st["token"] = torch.empty(R, dtype=torch.int32, device="cuda")
        st["prob"] = torch.empty(R, dtype=torch.float32, device="cuda")
    if own:                                        # the handles that a user's program keeps
        import paper_2604_07173_amd as L
        if case["op"] in ("share", "attend"):
            st["cache"] = L.KvCache(st["k"], st["v"])
            st["batch"] = L.KvBatch(st["start"], st["len"], st["table"], n_rows=T, max_rows=st["most"])
            st["shared"] = L.KvShared(case["seqs"], T)
            if case["op"] == "attend":             # once a step, for all layers
                L.lora_kv_share(st["cache"], st["batch"], st["shared"], max_rows=_MAX_ROWS)
                ws = L.lora_kv_attention_shared_ws_bytes(st["cache"], st["batch"], st["shared"], H)
                st["ws"] = torch.empty(max(256, ws), dtype=torch.uint8, device="cuda")
        elif case["op"] == "norm":
            st["norm"] = L.Norm(st["weight"], eps=_EPS, shift=case["shift"])
            st["rows8"] = L.Rows8(st["y8"], st["scale"], case["eight"]) if case["eight"] >= 0 else None
        else:
            st["how"] = L.Sampling(st["temperature"], st["top_k"], st["top_p"], st["min_p"])
    return st


def run(st):
    case = st["case"]
    return {"share": _share, "attend": _attend, "norm": _norm, "sample": _sample}[case["op"]](st, case)


# ---- which sequences hold the same first pages ---------------------------------------------------------


def _share(st, case):
    if own:
        import paper_2604_07173_amd as L
        sh = st["shared"]
        L.lora_kv_share(st["cache"], st["batch"], sh, max_rows=_MAX_ROWS)
        return dict(groups=sh.groups, rows=sh.rows, own=sh.own, place=sh.place, counts=sh.counts)
    n, page, T = case["seqs"], case["page"], st["n_rows"]
    table, start = st["table"].long(), st["start"].long()
    rows = start[1:] - start[:-1]
    whole = (st["len"].long() - rows) // page
    part = (rows >= 1) & (rows <= _MAX_ROWS) & (whole >= 1)
    key = table[:, 0]
    same = (key[:, None] == key) & part[:, None] & part
    lead = same.int().argmax(1)                      # the first of equals
    col = torch.arange(table.shape[1], device="cuda")
    common = ((table == table[lead]) & (col < torch.minimum(whole, whole[lead])[:, None])).long().cumprod(1).sum(1)
    joins = part & (common >= 1)
    to = torch.where(joins, lead, n)
    members = torch.zeros(n + 1, dtype=torch.long, device="cuda").scatter_add_(0, to, torch.ones_like(to))
    least = torch.full((n + 1,), 1 << 30, dtype=torch.long, device="cuda").scatter_reduce_(0, to, common, "amin")
    slots = torch.arange(n, device="cuda")
    heads = (lead == slots) & part & (members[:n] >= 2)
    number = heads.long().cumsum(0) - 1
    grouped = joins & (members[lead] >= 2)
    group = torch.where(grouped, number[lead], n)
    order = torch.argsort(group, stable=True)
    mine = torch.where(grouped, rows, 0)
    before = mine[order].cumsum(0) - mine[order]
    place = torch.where(grouped, torch.zeros_like(before).scatter_(0, order, before), -1)
    shared = torch.where(grouped, least[lead] * page, 0)
    # rows of groups, one group after another
    t = torch.arange(T, device="cuda")
    seq = torch.searchsorted(start, t, right=True) - 1
    at = torch.where(grouped[seq], place[seq] + t - start[seq], T)
    listed_rows = torch.full((T + 1,), -1, dtype=torch.long, device="cuda").scatter_(0, at, t)[:T]
    room = max(1, n // 2)
    where = torch.where(heads, number, room)
    total = torch.zeros(n + 1, dtype=torch.long, device="cuda").scatter_add_(0, torch.where(grouped, lead, n), mine)[:n]
    spread = lambda v, none: torch.full((room + 1,), none, dtype=torch.long, device="cuda").scatter_(0, where, v)[:room]     # noqa: E731
    groups = torch.stack([spread(slots, -1), spread(least[:n] * page, 0), spread(place, 0), spread(total, 0)], 1)
    groups[:, 1:] *= groups[:, :1] >= 0
    spared = (torch.where(heads, members[:n] - 1, 0) * torch.where(heads, least[:n] * page, 0)).sum().clamp(max=(1 << 31) - 1)
    counts = torch.stack([heads.sum(), mine.sum(), grouped.sum(), spared])
    return dict(groups=groups.int(), rows=listed_rows.int(), own=shared.int(), place=place.int(), counts=counts.int())


# ---- attention -----------------------------------------------------------------------------------------


def _attend(st, case):
    H, KV, D, page = case["heads"], case["kv"], case["dim"], case["page"]
    if own:
        import paper_2604_07173_amd as L
        L.lora_kv_attention_shared(st["cache"], 0, st["batch"], st["shared"], st["q"], H * D, H, st["out"], H * D, st["lse"],
                                   1.0 / math.sqrt(D), st["ws"], causal=case["causal"])
        return (st["out"], st["lse"]) if case["lse"] else (st["out"],)
    n, r, G = case["seqs"], st["most"], H // KV     # all sequences at once, padded to the longest and to `most` rows
    start, length = st["start"].long(), st["len"].long()
    count = start[1:] - start[:-1]
    i = torch.arange(r, device="cuda")
    at = (start[:-1, None] + torch.minimum(i, (count[:, None] - 1).clamp(min=0))).clamp(max=st["n_rows"] - 1)
    table = st["table"].long().clamp(min=0)
    tokens = table.shape[1] * page
    j = torch.arange(tokens, device="cuda")
    k = st["k"][0][table].transpose(1, 2).reshape(n, KV, tokens, D).float()
    q = st["q"][at].float().view(n, r, KV, G, D).transpose(1, 2).reshape(n, KV, r * G, D)
    s = torch.matmul(q * (1.0 / math.sqrt(D)), k.transpose(2, 3).contiguous()).view(n, KV, r, G, tokens)
    del k
    seen = j < length[:, None, None]
    if case["causal"]:
        seen = seen & (j <= (length - count)[:, None, None] + i[:, None])
    s = s.masked_fill(~seen.expand(n, r, tokens)[:, None, :, None, :], -math.inf)
    top = s.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, torch.zeros_like(top), top)
    p = (s - top).exp()
    del s
    total = p.sum(-1, keepdim=True)
    live = j < length[:, None]
    v = torch.where(live[:, None, :, None], st["v"][0][table].transpose(1, 2).reshape(n, KV, tokens, D).float(), torch.zeros((), device="cuda"))
    o = torch.matmul(p.view(n, KV, r * G, tokens), v).view(n, KV, r, G, D)
    o = (o / torch.where(total == 0, torch.ones_like(total), total)).transpose(1, 2).reshape(n * r, H * D)
    e = (top + total.log()).squeeze(-1).transpose(1, 2).reshape(n * r, H)
    mine = (i < count[:, None]).flatten()
    st["out"][at.flatten()[mine]] = o[mine].bfloat16()
    if case["lse"]:
        st["lse"][at.flatten()[mine]] = e[mine]
        return st["out"], st["lse"]
    return (st["out"],)


# ---- residual and norm ---------------------------------------------------------------------------------


def _norm(st, case):
    W, group = case["width"], case["eight"]
    if own:
        import paper_2604_07173_amd as L
        kind = lambda t: L.LORA_DTYPE_F32 if t is not None and t.dtype == torch.float32 else L.LORA_DTYPE_BF16     # noqa: E731
        L.lora_add_norm(st["norm"], case["rows"], st["x"], W, st["add"], W, st["sum"], W, st["y"], W, st["rows8"],
                        x_dtype=kind(st["x"]), add_dtype=kind(st["add"]))
    else:
        s = st["x"].float() if st["add"] is None else st["x"].float() + st["add"].float()
        st["sum"].copy_(s)
        y = s / (s.square().mean(-1, keepdim=True) + _EPS).sqrt() * (st["weight"].float() + case["shift"])
        if case["y"]:
            st["y"].copy_(y)
        if group >= 0:
            each = group or W
            over = -W % each
            blocks = (torch.cat([y, y.new_zeros((y.shape[0], over))], 1) if over else y).view(y.shape[0], -1, each)
            top = blocks.abs().amax(-1, keepdim=True)
            scale = torch.where(top == 0, torch.ones_like(top), top / _E4M3_MOST)
            st["y8"].copy_((blocks / scale).clamp(-_E4M3_MOST, _E4M3_MOST).view(y.shape[0], -1)[:, :W])
            st["scale"].copy_(scale.squeeze(-1))
    out = dict(sum=st["sum"])
    if case["y"]:
        out["y"] = st["y"]
    if group >= 0:
        out["y8"], out["scale"] = st["y8"], st["scale"]
    return out


# ---- the next token ------------------------------------------------------------------------------------


def _sample(st, case):
    R, V = case["rows"], case["vocab"]
    if own:
        import paper_2604_07173_amd as L
        L.lora_sample(st["logits"], V + case["pad"], R, V, st["how"], st["u"], st["token"], st["prob"],
                      dtype=L.LORA_DTYPE_F32 if case["f32"] else L.LORA_DTYPE_BF16)
        return st["token"], st["prob"]
    # in 64 bits: sums over the vocabulary decide between neighbouring tokens
    x = st["logits"][:, :V].double()
    T = st["temperature"].double()[:, None]
    value, index = torch.sort(x, dim=-1, descending=True, stable=True)
    w = ((value - value[:, :1]) / torch.where(T > 0, T, torch.ones_like(T))).exp()
    rank = torch.arange(V, device="cuda")
    k = st["top_k"].long()[:, None]
    w = w * ((k <= 0) | (rank < k))
    upto = w.cumsum(-1)
    top_p = st["top_p"].double()[:, None]
    keep = (top_p >= 1) | (upto - w < top_p * upto[:, -1:]) | (rank == 0)
    keep = keep & (w >= st["min_p"].double()[:, None]) & ((T > 0) | (rank == 0))
    w = torch.zeros_like(w).scatter_(1, index, w * keep)
    upto = w.cumsum(-1)
    total = upto[:, -1:]
    token = (upto <= st["u"].double()[:, None] * total).long().sum(-1, keepdim=True)
    last = torch.where(w > 0, rank, -1).amax(-1, keepdim=True)
    token = torch.minimum(token, last)
    st["token"].copy_(token[:, 0])
    st["prob"].copy_((w.gather(1, token) / total)[:, 0])
    return st["token"], st["prob"]


# ---- what a pass cannot do without, and the exact results ----------------------------------------------


def work(case):
    if case["op"] in ("share", "attend"):
        table, _ = _tables(case, np.random.RandomState(0))
        _, _, rows, lens = _lengths(case)
        # the groups by their definition, one sequence after another
        whole, led = (lens - rows) // case["page"], {}
        for q in np.nonzero((rows >= 1) & (rows <= _MAX_ROWS) & (whole >= 1))[0]:
            lead, members = led.setdefault(int(table[q, 0]), (q, []))
            differ = np.nonzero(table[q, :min(whole[q], whole[lead])] != table[lead, :min(whole[q], whole[lead])])[0]
            members.append(int(differ[0]) if len(differ) else int(min(whole[q], whole[lead])))
        groups = [(len(members), min(members) * case["page"]) for _, members in led.values() if len(members) >= 2]
        T, n = int(rows.sum()), len(lens)
        if case["op"] == "share":
            entries = sum(members * (tokens // case["page"]) for members, tokens in groups) + n
            return dict(bytes=4 * (entries + 2 * n + 2 * n + T + 4 * len(groups)), flops=entries)
        H, KV, D = case["heads"], case["kv"], case["dim"]
        tokens = int(lens[rows > 0].sum()) - sum((members - 1) * t for members, t in groups)
        pairs = int((rows * lens - (rows * (rows - 1) // 2 if case["causal"] else 0)).sum())
        return dict(bytes=tokens * KV * D * 4 + T * H * D * 4 + (T * H * 4 if case["lse"] else 0), flops=pairs * H * D * 4)
    if case["op"] == "norm":
        R, W = case["rows"], case["width"]
        each = 4 if case["f32"] else 2
        total = each + {"none": 0, "bf16": 2, "f32": 4}[case["add"]] + each + (2 if case["y"] else 0) + (case["eight"] >= 0)
        scales = (-(-W // case["eight"]) if case["eight"] else 1) if case["eight"] >= 0 else 0
        return dict(bytes=R * W * total + 2 * W + 4 * R * scales, flops=6 * R * W)
    return dict(bytes=case["rows"] * (case["vocab"] * (4 if case["f32"] else 2) + 28), flops=3 * case["rows"] * case["vocab"])


def exact(case, seed):
    if case["op"] == "share":
        return None                                  # numbers of slots, rows and tokens: nothing is computed in floating point
    global own
    mine, own = own, False
    try:
        st = prepare(case, seed)
    finally:
        own = mine
    if case["op"] == "norm":
        s = st["x"].double()
        if st["add"] is not None:
            s = s + st["add"].double()
        gain = st["weight"].double() + case["shift"]
        y = s * torch.rsqrt(torch.linalg.vector_norm(s, dim=1, keepdim=True) ** 2 / case["width"] + _EPS) * gain
        out = dict(sum=s)
        if case["y"]:
            out["y"] = y
        if case["eight"] >= 0:
            parts = y.split(case["eight"] or case["width"], dim=1)
            tops = [torch.linalg.vector_norm(p, ord=math.inf, dim=1, keepdim=True) for p in parts]
            scales = [torch.where(t > 0, t / _E4M3_MOST, torch.ones_like(t)) for t in tops]
            out["y8"] = torch.cat([p / t for p, t in zip(parts, scales)], 1)
            out["scale"] = torch.cat(scales, 1)
        return out
    if case["op"] == "sample":
        logits = st["logits"][:, :case["vocab"]].double().cpu().numpy()
        rules = [st[f].cpu().numpy() for f in ("temperature", "top_k", "top_p", "min_p", "u")]
        prob = np.zeros(case["rows"])
        for r in range(case["rows"]):
            T, k, p, least, u = (float(f[r]) for f in rules)
            row = logits[r]
            if T <= 0:
                prob[r] = 1.0
                continue
            order = np.argsort(-row, kind="stable")
            w = np.exp((row[order] - row.max()) / T)
            n = len(row) if k <= 0 else min(len(row), int(k))
            if p < 1:
                n = min(n, 1 + int(np.searchsorted(np.cumsum(w[:n]), p * w[:n].sum(), side="left")))
            n = max(1, min(n, int((w >= least).sum())))
            kept = np.sort(order[:n])
            w = np.exp((row[kept] - row.max()) / T)
            upto = np.cumsum(w)
            prob[r] = w[min(int(np.searchsorted(upto, u * upto[-1], side="right")), n - 1)] / upto[-1]
        return None, torch.from_numpy(prob)
    _, _, rows, lens = _lengths(case)
    H, KV, D, page = case["heads"], case["kv"], case["dim"], case["page"]
    G = H // KV
    out = torch.zeros((st["n_rows"], H, D), dtype=torch.float64, device="cuda")
    lse = torch.full((st["n_rows"], H), -math.inf, dtype=torch.float64, device="cuda")
    table = st["table"].cpu().numpy().astype(np.int64)
    starts = np.concatenate([[0], np.cumsum(rows)])
    for s, (r, n) in enumerate(zip(rows, lens)):
        if r == 0:
            continue
        pages = torch.from_numpy(table[s, :-(-n // page)]).cuda()
        at = slice(int(starts[s]), int(starts[s + 1]))
        hidden = torch.arange(n, device="cuda")[None, :] > torch.arange(n - r, n, device="cuda")[:, None]
        for h in range(KV):
            k = st["k"][0, pages, h].reshape(-1, D)[:n].double()
            v = st["v"][0, pages, h].reshape(-1, D)[:n].double()
            q = st["q"][at].view(-1, H, D)[:, h * G:(h + 1) * G].double().reshape(-1, D)
            score = (q @ k.t() / math.sqrt(D)).view(r, G, n)
            if case["causal"]:
                score = score.masked_fill(hidden[:, None, :], -math.inf)
            lse[at, h * G:(h + 1) * G] = torch.logsumexp(score, -1)
            out[at, h * G:(h + 1) * G] = (torch.softmax(score, -1).view(-1, n) @ v).view(r, G, D)
    out = out.view(-1, H * D)
    return (out, lse) if case["lse"] else (out,)
