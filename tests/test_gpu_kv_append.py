"""lora_rope_append against its definition in 64 bits: pairings, rotated widths, scaled frequencies, positions far
out and negative, input types and strides, pages, and what it must leave alone."""
import math

import numpy as np
import pytest
import torch

import paper_2604_07173_amd as L
from kv_common import KvCase

pytestmark = pytest.mark.gpu


def rotate64(x, pos, freq, rot, pairing, amplitude):
    """x [T][heads][D] in 64 bits, a pair as a complex number; also the pair's size, which bounds the errors."""
    x = x.clone()
    size = x.abs()
    a = torch.arange(rot // 2) if pairing == L.LORA_ROPE_HALF else torch.arange(0, rot, 2)
    b = a + (rot // 2 if pairing == L.LORA_ROPE_HALF else 1)
    turn = amplitude * torch.from_numpy(np.exp(1j * pos[:, None].astype(np.float64) * np.asarray(freq)[None]))[:, None]
    z = torch.complex(x[..., a], x[..., b]) * turn
    x[..., a], x[..., b] = z.real, z.imag
    size[..., a] = size[..., b] = z.abs()
    return x, size


def check(got, want, size):
    """One rounding to bf16 (half a step: 2^-8 of the value), and fp32 sine, cosine, products and one sum: 8 units of 2^-24 of the pair."""
    err = (got.double().cpu() - want).abs()
    bound = want.abs() * 2.0 ** -8 * 1.001 + size * 2.0 ** -21 + 1e-38
    assert (err <= bound).all(), f"worst {float((err / bound).max()):.2f}"


def run(rows, lens, heads=4, kv=2, dim=64, page=16, rot=None, pairing=L.LORA_ROPE_HALF, amplitude=1.0, f32=False, fused=False,
        slot_major=False, position=None, in_place=False, layers=1, layer=0, seed=0, parts="qkv", rope=True, **scaling):
    rot = dim if rot is None else rot
    case = KvCase(rows, lens, heads, kv, dim, page, slot_major, seed, stale=5.0, layers=layers).device()
    before = case.k5.clone(), case.v5.clone()
    g = torch.Generator().manual_seed(seed + 1)
    T, kind = case.T, torch.float32 if f32 else torch.bfloat16
    widths = [heads * dim, kv * dim, kv * dim]
    x = torch.randn((T, sum(widths) + 8), generator=g).to(kind)
    q, k, v = x[:, :widths[0]], x[:, widths[0]:widths[0] + widths[1]], x[:, -8 - widths[2]:-8]
    xd = x.cuda()
    qd, kd, vd = xd[:, :widths[0]], xd[:, widths[0]:widths[0] + widths[1]], xd[:, -8 - widths[2]:-8]
    if not fused:
        qd, kd, vd = qd.contiguous(), kd.contiguous(), vd.contiguous()
    q_out = qd if in_place else torch.full((T, widths[0] + 16), 9.0, dtype=torch.bfloat16, device="cuda")
    r = L.Rope(rot, pairing, amplitude, **scaling) if rope else None
    if position is not None:
        position = np.asarray(position, np.int32)
        case.batch = L.KvBatch(case.batch.row_start, case.batch.seq_len, case.batch.table, T, case.max_rows,
                               position=torch.from_numpy(position).cuda())
    has = lambda part, t: t if part in parts else None                            # noqa: E731
    L.lora_rope_append(case.cache, layer, case.batch, r, has("q", qd), qd.stride(0), has("k", kd), kd.stride(0), has("v", vd),
                       vd.stride(0), has("q", q_out), q_out.stride(0), heads, L.LORA_DTYPE_F32 if f32 else L.LORA_DTYPE_BF16)
    torch.cuda.synchronize()
    place = np.concatenate([np.arange(n - m, n) for m, n in zip(rows, lens)]) if T else np.zeros(0, np.int64)
    turn = place if position is None else position
    freq = L.lora_rope_freqs(rot, **scaling) if rope else [0.0] * (rot // 2)
    amp = amplitude if rope else 1.0
    if "q" in parts:
        want, size = rotate64(q.double().view(T, heads, dim), turn, freq, rot, pairing, amp)
        check(q_out[:, :widths[0]].reshape(T, heads, dim), want, size)
        if not in_place:
            assert (q_out[:, widths[0]:] == 9.0).all()
    after = [(t.transpose(2, 3) if slot_major else t).cpu() for t in (case.kd, case.vd)]
    if "k" in parts:
        want_k, size = rotate64(k.double().view(T, kv, dim), turn, freq, rot, pairing, amp)
        want_v = v.double().view(T, kv, dim)
        t = 0
        for s, (m, n) in enumerate(zip(rows, lens)):
            for p in range(n - m, n):
                at = (layer, case.table[s, p // page], slice(None), p % page) if p >= 0 else None
                if at:
                    check(after[0][at], want_k[t], size[t])
                    assert torch.equal(after[1][at], want_v[t].to(torch.bfloat16))
                    after[0][at], after[1][at] = before[0][at], before[1][at]
                t += 1
    assert torch.equal(after[0], before[0]) and torch.equal(after[1], before[1])      # nothing else was touched
    return case, q_out


@pytest.mark.parametrize("pairing", [L.LORA_ROPE_HALF, L.LORA_ROPE_INTERLEAVED])
@pytest.mark.parametrize("dim,rot", [(64, 64), (128, 128), (128, 64), (128, 32), (80, 48), (80, 20), (96, 24), (40, 40), (8, 8), (8, 2),
                                     (256, 256), (64, 6), (72, 16), (64, 62)])
@pytest.mark.parametrize("f32", [False, True])
def test_pairings_and_widths(pairing, dim, rot, f32):
    run([3, 0, 1, 7], [40, 5, 17, 7], dim=dim, rot=rot, pairing=pairing, f32=f32, fused=not f32)


@pytest.mark.parametrize("page", [1, 8, 16, 64, 1024])
@pytest.mark.parametrize("slot_major", [False, True])
def test_pages(page, slot_major):
    run([5, 30, 1], [5, 70, 33], page=page, slot_major=slot_major, fused=True)


@pytest.mark.parametrize("scaling", [dict(), dict(scaling=L.LORA_ROPE_LINEAR, factor=4.0), dict(scaling=L.LORA_ROPE_BASE, factor=8.0),
                                     dict(scaling=L.LORA_ROPE_PARTS, base=5e5, factor=8.0, original_len=8192.0, low=1.0, high=4.0)])
@pytest.mark.parametrize("amplitude", [1.0, 1.2079])
def test_far_positions(scaling, amplitude):
    """The angle of a position of a million is as exact as that of the first."""
    position = [0, 1, -1, 131071, 1000003, -999983, 2 ** 31 - 1, -2 ** 31, 77]
    run([4, 5], [30, 12], dim=128, amplitude=amplitude, position=position, **scaling)


def test_negated_positions_undo_it():
    case, q_out = run([50], [400], dim=128)
    pos = torch.arange(350, 400, dtype=torch.int32, device="cuda")
    back = torch.empty((50, 4 * 128), dtype=torch.bfloat16, device="cuda")
    g = torch.Generator().manual_seed(1)
    x = torch.randn((50, 4 * 128 + 4 * 128 + 8), generator=g).to(torch.bfloat16)[:, :512]
    batch = L.KvBatch(case.batch.row_start, case.batch.seq_len, case.batch.table, 50, position=-pos)
    L.lora_rope_append(case.cache, 0, batch, L.Rope(128), q_out, q_out.stride(0), None, 0, None, 0, back, 512, 4)
    # two roundings of a pair of size s: each at most 2^-8 of a component, turned into the other
    size = (x.double() ** 2).view(50, 4, 2, 64).sum(2, keepdim=True).sqrt().expand(50, 4, 2, 64).reshape(50, 512)
    assert ((back.double().cpu() - x.double()).abs() <= size * 2.0 ** -8 * 2.5).all()


@pytest.mark.parametrize("pairing", [L.LORA_ROPE_HALF, L.LORA_ROPE_INTERLEAVED])
@pytest.mark.parametrize("rot", [128, 32, 20])
def test_in_place(pairing, rot):
    run([3, 9], [40, 9], dim=128, rot=rot, pairing=pairing, in_place=True, fused=True)


@pytest.mark.parametrize("parts", ["q", "kv"])
@pytest.mark.parametrize("rope", [True, False])
def test_parts(parts, rope):
    run([3, 9], [40, 9], parts=parts, rope=rope)


def test_one_row_and_many():
    run([1], [1])
    run([1] * 200, list(range(1, 201)), page=8)
    run([600, 1, 0, 300], [1000, 900, 40, 300], heads=2, kv=1)


def test_wide_layers():
    run([2, 3], [20, 30], heads=40, kv=8, dim=128, layers=3, layer=1)
    run([2], [20], heads=3, kv=3, dim=256, rot=64)


def test_rows_before_the_start_are_not_written():
    case, _ = run([5], [3])
    assert int(case.batch.status.item()) == L.LORA_STATUS_BAD_LENGTH


def test_pages_outside_the_cache_are_not_written():
    case = KvCase([2, 2], [20, 20], stale=5.0).device()
    case.batch.table[0, 1] = case.n_pages
    k = torch.ones((4, 128), dtype=torch.bfloat16, device="cuda")
    want = case.kd.clone()
    want[0, case.table[1, 1], :, 2:4] = 1.0
    L.lora_rope_append(case.cache, 0, case.batch, None, None, 0, k, 128, k, 128, None, 0, 0)
    torch.cuda.synchronize()
    assert int(case.batch.status.item()) == L.LORA_STATUS_BAD_PAGE
    assert torch.equal(case.kd, want)


def test_no_rows():
    case = KvCase([0], [5]).device()
    L.lora_rope_append(case.cache, 0, case.batch, None, None, 0, case.kd, 128, case.kd, 128, None, 0, 0)


def test_in_a_graph():
    case = KvCase([1] * 20, list(range(30, 50)), dim=128, stale=0.0).device()
    x = torch.randn((20, 8 * 128), device="cuda").bfloat16()
    out = torch.zeros((20, 512), dtype=torch.bfloat16, device="cuda")
    rope = L.Rope(128)
    call = lambda: L.lora_rope_append(case.cache, 0, case.batch, rope, x, 1024, x[:, 512:], 1024, x[:, 768:], 1024, out, 512, 4)  # noqa: E731
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for _ in range(3):
        x.normal_()
        case.batch.seq_len.sub_(1)
        call()
        want = out.clone(), case.kd.clone(), case.vd.clone()
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want[0]) and torch.equal(case.kd, want[1]) and torch.equal(case.vd, want[2])
