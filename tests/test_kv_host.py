"""Paged cache without a GPU: what the calls refuse before any device work, and the rotary frequencies."""
import ctypes as C
import math

import pytest

import paper_2604_07173_amd as L
from paper_2604_07173_amd import binding as B

OK, INVALID, SHAPE, SMALL, MISALIGNED, LARGE = 0, -1, -2, -4, -7, -8
A = 0x10000                                    # an aligned address that is never looked at


@pytest.fixture(scope="module")
def lib():
    return L.load_library()


def cache(**kw):
    """2 layers of 10 pages, 4 heads x 16 tokens x 64."""
    d = dict(k=A, v=A, n_layers=2, n_pages=10, n_heads=4, page_size=16, head_dim=64, layer_stride=40960, page_stride=4096,
             head_stride=1024, token_stride=64)
    d.update(kw)
    return C.byref(B._KvCache(**d))


def batch(**kw):
    d = dict(n_seqs=3, n_rows=5, max_rows=2, max_pages=4, row_start=A, seq_len=A, table=A, position=None, status=A)
    d.update(kw)
    return C.byref(B._KvBatch(**d))


def append(lib, c=None, layer=0, b=None, rope=None, q=A, ldq=512, k=A, ldk=256, v=A, ldv=256, qo=2 * A, ldqo=512, heads=8, dtype=0):
    return lib.lora_rope_append(cache() if c is None else c, layer, batch(n_rows=0) if b is None else b, rope, q, ldq, k, ldk, v,
                                ldv, qo, ldqo, heads, dtype, None)


def attend(lib, c=None, layer=0, b=None, q=A, ldq=512, heads=8, out=2 * A, ldo=512, lse=None, scale=0.125, causal=1, window=0, ws=A,
           ws_bytes=1 << 30):
    return lib.lora_kv_attention(cache() if c is None else c, layer, batch(n_rows=0) if b is None else b, q, ldq, heads, out, ldo,
                                 lse, scale, causal, window, ws, ws_bytes, None)


BAD_CACHES = [
    (dict(k=None), INVALID), (dict(v=None), INVALID), (dict(k=A + 8), MISALIGNED), (dict(v=A + 2), MISALIGNED),
    (dict(n_layers=0), INVALID), (dict(n_pages=0), INVALID), (dict(n_heads=-1), INVALID), (dict(page_size=0), SHAPE),
    (dict(page_size=24), SHAPE), (dict(page_size=2048), SHAPE), (dict(head_dim=4), SHAPE), (dict(head_dim=60), SHAPE),
    (dict(head_dim=264), SHAPE), (dict(token_stride=56), SHAPE), (dict(token_stride=68), SHAPE), (dict(head_stride=1016), SHAPE),
    (dict(page_stride=4088), SHAPE), (dict(layer_stride=40952), SHAPE), (dict(page_stride=-4096), SHAPE), (dict(n_layers=20000), LARGE),
]


@pytest.mark.parametrize("change,status", BAD_CACHES)
def test_caches_that_are_refused(lib, change, status):
    c = cache(**change)
    assert append(lib, c=c) == status and attend(lib, c=c) == status
    moves = C.byref(B._KvMoves(100, 0, A, A, A, A, 1 << 20))
    state, to = (C.byref(B._KvState(3, 4, a, a, None)) for a in (A, 2 * A))
    assert lib.lora_kv_plan(c, state, to, A, A, moves, None) == status
    assert lib.lora_kv_compact(c, state, to, moves, None) == status
    assert lib.lora_kv_copy_pages(c, moves, 0, None) == status
    assert lib.lora_kv_attention_ws_bytes(c, batch(), 8) == 0


@pytest.mark.parametrize("change", [
    dict(), dict(head_stride=64, token_stride=256),                                         # [token][head]
    dict(layer_stride=4096, page_stride=8192),                                              # layers inside a page
    dict(token_stride=72, head_stride=16 * 72, page_stride=5000, layer_stride=50000),       # holes
    dict(n_heads=1, head_stride=0), dict(n_layers=1, layer_stride=0), dict(page_size=1, token_stride=0, head_stride=64)])
def test_caches_that_are_taken(lib, change):
    assert append(lib, c=cache(**change), q=None) == OK and attend(lib, c=cache(**change)) in (OK, OK)
    assert lib.lora_kv_attention_ws_bytes(cache(**change), batch(), 8) > 0


@pytest.mark.parametrize("change,status", [
    (dict(n_seqs=0), INVALID), (dict(n_seqs=-1), INVALID), (dict(n_rows=-1), INVALID), (dict(max_rows=-1), INVALID),
    (dict(max_pages=0), INVALID), (dict(row_start=None), INVALID), (dict(seq_len=None), INVALID), (dict(table=None), INVALID),
    (dict(status=None), INVALID), (dict(n_rows=L.LORA_MAX_ROWS_LONG + 1), LARGE), (dict(n_seqs=L.LORA_MAX_ROWS_LONG + 1), LARGE)])
def test_batches_that_are_refused(lib, change, status):
    b = batch(**change)
    assert append(lib, b=b) == status and attend(lib, b=b) == status
    assert lib.lora_rope_append(cache(), 0, None, None, A, 512, A, 256, A, 256, 2 * A, 512, 8, 0, None) == INVALID
    assert lib.lora_kv_attention(cache(), 0, None, A, 512, 8, A, 512, None, 1.0, 1, 0, A, 1, None) == INVALID


@pytest.mark.parametrize("change,status", [
    (dict(layer=2), SHAPE), (dict(layer=-1), SHAPE), (dict(dtype=2), INVALID), (dict(k=None), INVALID), (dict(v=None), INVALID),
    (dict(q=None, k=None, v=None), INVALID), (dict(q=A + 8), MISALIGNED), (dict(k=A + 8), MISALIGNED), (dict(v=A + 4), MISALIGNED),
    (dict(qo=A + 8), MISALIGNED), (dict(qo=None), INVALID), (dict(ldq=504), SHAPE), (dict(ldq=516), SHAPE), (dict(ldk=248), SHAPE),
    (dict(ldv=260), SHAPE), (dict(ldqo=504), SHAPE), (dict(heads=0), SHAPE), (dict(qo=A, ldqo=520), INVALID),
    (dict(qo=A, dtype=1), INVALID)])
def test_appends_that_are_refused(lib, change, status):
    assert append(lib, b=batch(), **change) == status


@pytest.mark.parametrize("change,status", [
    (dict(freq=None), INVALID), (dict(freq=A + 4), MISALIGNED), (dict(rot_dim=0), SHAPE), (dict(rot_dim=7), SHAPE),
    (dict(rot_dim=66), SHAPE), (dict(pairing=2), INVALID), (dict(amplitude=math.inf), INVALID), (dict(amplitude=math.nan), INVALID)])
def test_rotations_that_are_refused(lib, change, status):
    d = dict(freq=A, rot_dim=64, pairing=0, amplitude=1.0, reserved=0)
    d.update(change)
    assert append(lib, b=batch(), rope=C.byref(B._Rope(**d))) == status


@pytest.mark.parametrize("change,status", [
    (dict(layer=2), SHAPE), (dict(heads=6), SHAPE), (dict(heads=0), SHAPE), (dict(heads=4 * 65), SHAPE), (dict(scale=0.0), INVALID),
    (dict(scale=-1.0), INVALID), (dict(scale=math.nan), INVALID), (dict(scale=math.inf), INVALID), (dict(window=-1), INVALID),
    (dict(window=5, causal=0), INVALID), (dict(q=None), INVALID), (dict(out=None), INVALID), (dict(q=A + 8), MISALIGNED),
    (dict(out=A + 8), MISALIGNED), (dict(ldq=504), SHAPE), (dict(ldo=516), SHAPE), (dict(ws=None), INVALID), (dict(ws=A + 8), MISALIGNED),
    (dict(lse=A + 2), MISALIGNED), (dict(out=A), INVALID), (dict(ws_bytes=16), SMALL)])
def test_attentions_that_are_refused(lib, change, status):
    assert attend(lib, b=batch(), **change) == status


def test_workspace_queries(lib):
    need = lib.lora_kv_attention_ws_bytes(cache(), batch(), 8)
    assert need > 0 and attend(lib, b=batch(), ws_bytes=need - 1) == SMALL
    assert lib.lora_kv_attention_ws_bytes(cache(), batch(n_rows=500, max_rows=300), 8) >= need
    for heads in (0, 6, 4 * 65, -4):
        assert lib.lora_kv_attention_ws_bytes(cache(), batch(), heads) == 0
    assert lib.lora_kv_attention_ws_bytes(cache(), None, 8) == 0
    assert lib.lora_kv_moves_ws_bytes(0, 4) == 0 and lib.lora_kv_moves_ws_bytes(4, 0) == 0 and lib.lora_kv_moves_ws_bytes(4, 4) > 0


def test_page_calls_that_are_refused(lib):
    def call(compact=False, c=None, src=A, new=A, fro=None, to=None, **kw):
        f, t = (dict(n_seqs=3, max_pages=4, table=a, seq_len=a + 64, page_ref=a + 128) for a in (A, 2 * A))
        f.update(fro or {})
        t.update(to or {})
        m = dict(capacity=5, reserved=0, pairs=A, counts=A, status=A, ws=A, ws_bytes=lib.lora_kv_moves_ws_bytes(10, 3))
        m.update(kw)
        args = [cache(), C.byref(B._KvState(**f)), C.byref(B._KvState(**t))]
        if compact:
            return lib.lora_kv_compact(*args, C.byref(B._KvMoves(**m)), None)
        return lib.lora_kv_plan(*args, src, new, C.byref(B._KvMoves(**m)), None)

    for compact in (False, True):
        for change, status in ((dict(fro=dict(table=None)), INVALID), (dict(to=dict(seq_len=None)), INVALID), (dict(fro=dict(n_seqs=0)), INVALID),
                               (dict(to=dict(n_seqs=4)), SHAPE), (dict(to=dict(max_pages=5)), SHAPE), (dict(to=dict(table=A)), INVALID),
                               (dict(to=dict(seq_len=A + 64)), INVALID), (dict(to=dict(page_ref=A + 128)), INVALID),
                               (dict(pairs=None), INVALID), (dict(counts=None), INVALID), (dict(status=None), INVALID),
                               (dict(ws=None), INVALID), (dict(ws=A + 4), MISALIGNED), (dict(capacity=2), SMALL),
                               (dict(ws_bytes=64), SMALL)):
            assert call(compact, **change) == status, (compact, change)
    assert call(src=None) == INVALID and call(new=None) == INVALID
    args = [cache(), C.byref(B._KvState(3, 4, A, A, None)), C.byref(B._KvState(3, 4, 2 * A, 2 * A, None))]
    assert lib.lora_kv_plan(*args, A, A, None, None) == INVALID and lib.lora_kv_plan(None, *args[1:], A, A, None, None) == INVALID
    copy = lambda n, **kw: lib.lora_kv_copy_pages(cache(), C.byref(B._KvMoves(**dict(dict(capacity=5, pairs=A, counts=A), **kw))), n, None)  # noqa: E731
    assert copy(-1) == INVALID and copy(6) == SMALL and copy(0) == OK and copy(2, pairs=None) == INVALID and copy(2, counts=None) == INVALID
    assert lib.lora_kv_copy_pages(cache(), None, 1, None) == INVALID


def test_frequencies():
    plain = L.lora_rope_freqs(64)
    assert plain[0] == 1.0 and len(plain) == 32
    for i, f in enumerate(plain):
        assert f == pytest.approx(10000.0 ** (-i / 32), rel=1e-14)
    assert L.lora_rope_freqs(64, scaling=L.LORA_ROPE_LINEAR, factor=4.0) == pytest.approx([f / 4 for f in plain], rel=1e-14)
    # the base form leaves the fastest pair alone and slows the slowest one by the whole factor
    base = L.lora_rope_freqs(64, scaling=L.LORA_ROPE_BASE, factor=4.0)
    assert base[0] == 1.0 and base[31] == pytest.approx(plain[31] / 4, rel=1e-12)
    assert L.lora_rope_freqs(2, scaling=L.LORA_ROPE_BASE, factor=4.0) == [1.0]
    parts = L.lora_rope_freqs(128, base=5e5, scaling=L.LORA_ROPE_PARTS, factor=8.0, original_len=8192.0, low=1.0, high=4.0)
    for i, f in enumerate(parts):
        full = 5e5 ** (-i / 64)
        turns = 8192 * full / (2 * math.pi)
        g = min(1.0, max(0.0, (turns - 1) / 3))
        assert f == pytest.approx(g * full + (1 - g) * full / 8, rel=1e-12)
    assert parts[0] == 1.0 and parts[63] == pytest.approx(5e5 ** (-63 / 64) / 8, rel=1e-12)


@pytest.mark.parametrize("change,status", [
    (dict(rot_dim=0), SHAPE), (dict(rot_dim=5), SHAPE), (dict(rot_dim=258), SHAPE), (dict(base=1.0), INVALID), (dict(base=math.nan), INVALID),
    (dict(factor=0.5), INVALID), (dict(factor=math.inf), INVALID), (dict(scaling=4), INVALID), (dict(scaling=-1), INVALID),
    (dict(scaling=3, original_len=0.0), INVALID), (dict(scaling=3, original_len=8.0, low=2.0, high=2.0), INVALID),
    (dict(scaling=3, original_len=8.0, low=-1.0, high=2.0), INVALID)])
def test_frequencies_that_are_refused(change, status):
    args = dict(rot_dim=64, base=1e4, scaling=0, factor=1.0, original_len=0.0, low=0.0, high=0.0)
    args.update(change)
    with pytest.raises(L.LoraError) as e:
        L.lora_rope_freqs(**args)
    assert e.value.status == status
    assert L.load_library().lora_rope_freqs(None, None) == INVALID


def test_handles_check_their_tensors():
    import torch
    k = torch.empty((1, 4, 2, 16, 64), dtype=torch.bfloat16)
    for bad in (k[0], k.float(), k[..., ::2], k[:, :2]):
        with pytest.raises(ValueError):
            L.KvCache(bad, k)
    c = L.KvCache(k.transpose(2, 3).contiguous().transpose(2, 3), k.transpose(2, 3).contiguous().transpose(2, 3)).c
    assert (c.n_heads, c.page_size, c.token_stride, c.head_stride) == (2, 16, 128, 64)
    i = torch.zeros(3, dtype=torch.int32)
    with pytest.raises(ValueError):
        L.KvBatch(i, i, torch.zeros((3, 2), dtype=torch.int32), 3)              # row_start needs one more
    with pytest.raises(ValueError):
        L.KvBatch(torch.zeros(4, dtype=torch.int64), i, torch.zeros((3, 2), dtype=torch.int32), 3)
    with pytest.raises(ValueError):
        L.KvState(torch.zeros((3, 4), dtype=torch.int32)[:, ::2], i)
