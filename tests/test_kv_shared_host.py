"""Sequences that share pages, without a GPU: what the calls refuse, every argument's way through the extension module, and the grid of
long tiles (compiled for the CPU with g++)."""
import ctypes as C
import os
import subprocess
import tempfile

import numpy as np
import pytest

import paper_2604_07173_amd as L
from paper_2604_07173_amd import binding as B
from test_kv_host import A, BAD_CACHES, INVALID, LARGE, MISALIGNED, OK, SHAPE, SMALL, batch, cache
from test_kv_pycall import Buffer, Holder

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def lib():
    return L.load_library()


def shared(**kw):
    d = dict(n_seqs=3, n_rows=5, max_group_rows=0, groups=A, rows=A, own=A, place=A, counts=A, ws=A, ws_bytes=1 << 20)
    d.update(kw)
    return C.byref(B._KvShared(**d))


def share(lib, c=None, b=None, sh=None, min_pages=1, max_rows=0):
    return lib.lora_kv_share(cache() if c is None else c, batch(n_rows=0) if b is None else b, shared() if sh is None else sh, min_pages, max_rows, None)


def attend(lib, c=None, layer=0, b=None, sh=None, q=A, ldq=512, heads=8, out=2 * A, ldo=512, lse=None, scale=0.125, causal=1, ws=A,
           ws_bytes=1 << 30):
    return lib.lora_kv_attention_shared(cache() if c is None else c, layer, batch(n_rows=0) if b is None else b, shared() if sh is None else sh,
                                        q, ldq, heads, out, ldo, lse, scale, causal, ws, ws_bytes, None)


@pytest.mark.parametrize("change,status", BAD_CACHES)
def test_caches_that_are_refused(lib, change, status):
    assert share(lib, c=cache(**change)) == status and attend(lib, c=cache(**change)) == status
    assert lib.lora_kv_attention_shared_ws_bytes(cache(**change), batch(), shared(), 8) == 0


@pytest.mark.parametrize("change,status", [
    (dict(n_seqs=0), INVALID), (dict(n_rows=-1), INVALID), (dict(max_pages=0), INVALID), (dict(row_start=None), INVALID),
    (dict(seq_len=None), INVALID), (dict(table=None), INVALID), (dict(status=None), INVALID), (dict(n_rows=L.LORA_MAX_ROWS_LONG + 1), LARGE)])
def test_batches_that_are_refused(lib, change, status):
    assert share(lib, b=batch(**change)) == status and attend(lib, b=batch(**change)) == status


@pytest.mark.parametrize("change,status", [
    (dict(n_seqs=-1), INVALID), (dict(n_rows=-1), INVALID), (dict(max_group_rows=-1), INVALID), (dict(groups=None), INVALID), (dict(rows=None), INVALID),
    (dict(own=None), INVALID), (dict(place=None), INVALID), (dict(counts=None), INVALID), (dict(n_seqs=4), SHAPE), (dict(n_seqs=2), SHAPE),
    (dict(n_rows=L.LORA_MAX_ROWS_LONG + 1), LARGE)])
def test_groups_that_are_refused(lib, change, status):
    assert share(lib, b=batch(), sh=shared(**change)) == status and attend(lib, b=batch(), sh=shared(**change)) == status


@pytest.mark.parametrize("change,kw,status", [
    (dict(ws=None), {}, INVALID), (dict(ws=A + 4), {}, MISALIGNED), (dict(ws_bytes=64), {}, SMALL), (dict(n_rows=4), {}, SMALL),
    (dict(n_rows=2), dict(max_rows=1), SMALL), ({}, dict(min_pages=0), INVALID), ({}, dict(max_rows=-1), INVALID)])
def test_searches_that_are_refused(lib, change, kw, status):
    assert share(lib, b=batch(), sh=shared(**change), **kw) == status


@pytest.mark.parametrize("change,status", [
    (dict(layer=2), SHAPE), (dict(layer=-1), SHAPE), (dict(heads=6), SHAPE), (dict(heads=0), SHAPE), (dict(heads=4 * 65), SHAPE),
    (dict(scale=0.0), INVALID), (dict(scale=float("nan")), INVALID), (dict(scale=float("inf")), INVALID), (dict(q=None), INVALID),
    (dict(out=None), INVALID), (dict(q=A + 8), MISALIGNED), (dict(out=A + 8), MISALIGNED), (dict(ldq=504), SHAPE), (dict(ldo=516), SHAPE),
    (dict(ws=None), INVALID), (dict(ws=A + 8), MISALIGNED), (dict(lse=A + 2), MISALIGNED), (dict(out=A), INVALID), (dict(ws_bytes=16), SMALL)])
def test_attentions_that_are_refused(lib, change, status):
    assert attend(lib, b=batch(), **change) == status


def test_sizes(lib):
    need = lib.lora_kv_attention_shared_ws_bytes(cache(), batch(), shared(), 8)
    assert need > 0 and attend(lib, b=batch(), ws_bytes=need - 1) == SMALL
    assert lib.lora_kv_attention_shared_ws_bytes(cache(), batch(), shared(n_rows=50), 8) > need
    assert lib.lora_kv_attention_shared_ws_bytes(cache(), batch(), None, 8) == 0
    assert lib.lora_kv_attention_shared_ws_bytes(cache(), batch(), shared(), 6) == 0
    rows = 1 << 20                                   # rows x heads: at most 2^26
    big = batch(n_rows=rows, n_seqs=3)
    assert lib.lora_kv_attention_shared_ws_bytes(cache(), big, shared(n_rows=rows), 64) > 0
    assert lib.lora_kv_attention_shared_ws_bytes(cache(), big, shared(n_rows=rows), 68) == 0
    assert attend(lib, b=big, sh=shared(n_rows=rows), heads=68, ldq=68 * 64, ldo=68 * 64) == LARGE
    assert attend(lib, b=batch(), sh=shared(n_rows=rows), heads=68, ldq=68 * 64, ldo=68 * 64) == LARGE
    assert lib.lora_kv_share_ws_bytes(0) == 0 and lib.lora_kv_share_ws_bytes(L.LORA_MAX_ROWS_LONG + 1) == 0
    assert lib.lora_kv_share_ws_bytes(L.LORA_MAX_ROWS_LONG) > 0


def test_empty_batches_are_done_at_once(lib):
    assert share(lib) == OK and attend(lib) == OK
    assert attend(lib, q=None, out=None, ws=None) == OK


def test_every_argument_arrives_where_ctypes_puts_it():
    b = [Buffer(1000 + i, 0x7F0000000000 + 4096 * i) for i in range(4)]
    a = [v.address for v in b]
    big = 1 << 40
    lib = L.load_library()
    names = ("lora_kv_share", "lora_kv_attention_shared")
    calls, keep, addresses, through = [], [], {}, {}
    for name in names:
        types = getattr(lib, name).argtypes

        def note(*args, name=name, types=types):
            calls.append((name, [C.addressof(v.contents) if v and issubclass(t, C._Pointer) else None if issubclass(t, C._Pointer) else v
                                 for t, v in zip(types, args)]))
            return 0

        proto = C.CFUNCTYPE(C.c_int, *types)
        keep.append(proto(note))
        addresses[name] = C.cast(keep[-1], C.c_void_p).value
        through[name] = proto(addresses[name])
    c, t, s = (Holder(x()) for x in (B._KvCache, B._KvBatch, B._KvShared))
    r = lambda h: C.byref(h.c)                                                  # noqa: E731
    B._calls().bind_shared(addresses)
    try:
        for short, long_way in [
            (lambda: L.lora_kv_share(c, t, s, 4, 6, stream=9), lambda: through["lora_kv_share"](r(c), r(t), r(s), 4, 6, 9)),
            (lambda: L.lora_kv_attention_shared(c, 3, t, s, b[0], 8, 32, b[1], big, b[2], 0.125, b[3], causal=False, stream=9),
             lambda: through["lora_kv_attention_shared"](r(c), 3, r(t), r(s), a[0], 8, 32, a[1], big, a[2], 0.125, 0, a[3], 2006, 9)),
        ]:
            short()
            assert long_way() == 0
            (name, got), (name2, want) = calls[-2:]
            assert name == name2 and got == want, name
    finally:
        B._calls().bind_shared({n: C.cast(getattr(lib, n), C.c_void_p).value for n in names})
    with pytest.raises(L.LoraError):                  # converted, then refused for the empty cache
        L.lora_kv_share(c, t, s, stream=0)
    with pytest.raises(AttributeError):
        L.lora_kv_share(c, t, b[0], stream=0)
    with pytest.raises(OverflowError):
        L.lora_kv_share(c, t, s, min_pages=1 << 40, stream=0)


SRC = r'''
#include <cstdio>
#include "kv_work.h"
int main()
{
    int a[7];
    while (scanf("%d %d %d %d %d %d %d", a, a + 1, a + 2, a + 3, a + 4, a + 5, a + 6) == 7) {
        const lora::SharedKinds k = lora::shared_kinds_of(a[0], a[1], a[2], a[3], a[4], a[5], a[6], 64);
        printf("%d %d %d %lld\n", k.has_long, k.limit, k.group_limit, (long long)k.long_items);
    }
    printf("%d %d %d %lld %d\n", lora::kLongTile, lora::kLongTarget, lora::kLongMinSplit, (long long)lora::kSharedRowsHeads, lora::kSharedTarget);
    return 0;
}
'''


def test_there_is_a_workgroup_for_every_item_and_no_launch_is_too_large():
    with tempfile.TemporaryDirectory() as d:
        src, exe = os.path.join(d, "probe.cpp"), os.path.join(d, "probe")
        open(src, "w").write(SRC)
        subprocess.check_call(["g++", "-O1", "-std=c++17", "-I", os.path.join(ROOT, "paper_2604_07173_amd", "csrc"), src, "-o", exe])
        rng = np.random.default_rng(7)
        cases, batches = [], []
        for _ in range(3000):
            kv = int(rng.choice([1, 2, 8]))
            heads = kv * int(rng.choice([1, 2, 4, 5, 17, 64]))
            n = int(2 ** rng.uniform(1, 9))
            rows = rng.integers(0, int(rng.choice([2, 5, 80])), n)
            rows[0] = 1
            of = rng.integers(0, int(rng.integers(1, n + 1)), n)
            group_rows = np.array([rows[of == g].sum() for g in np.unique(of) if (of == g).sum() > 1], dtype=np.int64)
            room = int(rng.choice([rows.sum(), max(1, group_rows.sum())]))
            cases.append((n, int(rows.sum()), int(rng.choice([0, rows.max(), 1])), room, int(rng.choice([0, 1, max(1, group_rows.max(initial=1))])), heads, kv))
            lens = (2 ** rng.uniform(0, 15, n + len(group_rows))).astype(np.int64)
            batches.append((np.concatenate([rows, group_rows]), n, lens))
        big = [(n, rows, 0, rows, 0, 64, kv) for rows in (1 << 20, 1 << 19) for n in (1, 2, 1 << 20) for kv in (1, 64)]
        text = "\n".join(" ".join(map(str, c)) for c in cases + big)
        lines = subprocess.run([exe], input=text, capture_output=True, text=True, check=True).stdout.split("\n")
    got = [tuple(map(int, l.split())) for l in lines if l]
    tile, target, split, most, shared = got.pop()
    assert most == 1 << 26
    for c, (rows, n, lens), (has_long, limit, group_limit, items) in zip(cases, batches, got):
        if not has_long:
            continue
        kv, group = c[6], c[5] // c[6]
        r = rows * group
        limits = np.where(np.arange(len(rows)) < n, limit, group_limit)
        tiles = np.where(r > limits, -(-r // tile), 0)
        whole, half = float((tiles * lens).sum()) * kv, 0.5 * float(tiles.sum()) * kv
        each = whole / max(shared - half, 0.5 * shared)
        if each < split:
            each = whole / max(target - half, 0.5 * target)
        chunk = split if each < split else (int(each) + 128) >> 7 << 7
        cuts = np.where(lens <= chunk, 1, -(-lens // chunk))
        assert int((tiles * cuts).sum()) * kv <= items, c
        # partial results: of cut tiles only
        assert int((tiles * cuts)[cuts > 1].sum()) * kv <= 2 * shared, c
    for c, g in zip(big, got[len(cases):]):
        assert 0 < g[3] * 256 < 1 << 32, (c, g)
