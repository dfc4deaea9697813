"""Residual norm and sampling without a GPU: what the calls and the handles refuse, and every argument's way through the extension
module."""
import ctypes as C

import pytest
import torch

import paper_2604_07173_amd as L
from paper_2604_07173_amd import binding as B
from test_kv_pycall import Buffer, Holder

OK, INVALID, SHAPE, MISALIGNED, LARGE = 0, -1, -2, -7, -8
A = 0x10000                                    # aligned addresses that are never looked at


@pytest.fixture(scope="module")
def lib():
    return L.load_library()


def norm(lib, n=4, x=A, ldx=64, xt=0, add=2 * A, lda=64, at=0, total=3 * A, lds=64, out=4 * A, ldo=64, r8=None, **kw):
    d = dict(weight=A, width=64, weight_dtype=0, eps=1e-5, shift=0.0)
    d.update(kw)
    return lib.lora_add_norm(C.byref(B._Norm(**d)), n, x, ldx, xt, add, lda, at, total, lds, out, ldo, r8, None)


def rows8(**kw):
    d = dict(values=5 * A, scale=6 * A, ld=64, ld_scale=8, group=16, reserved=0)
    d.update(kw)
    return C.byref(B._Rows8(**d))


@pytest.mark.parametrize("change,status", [
    (dict(n=-1), INVALID), (dict(n=L.LORA_NORM_MAX_ROWS + 1), LARGE), (dict(width=0), SHAPE), (dict(width=12), SHAPE), (dict(width=-8), SHAPE),
    (dict(width=L.LORA_NORM_MAX_WIDTH + 8), LARGE), (dict(weight_dtype=2), INVALID), (dict(xt=2), INVALID), (dict(at=-1), INVALID), (dict(eps=0.0), INVALID),
    (dict(eps=-1e-5), INVALID), (dict(eps=1e-42), INVALID), (dict(eps=float("nan")), INVALID), (dict(eps=float("inf")), INVALID),
    (dict(shift=float("inf")), INVALID), (dict(weight=A + 8), MISALIGNED), (dict(x=None), INVALID), (dict(x=A + 8), MISALIGNED), (dict(ldx=56), SHAPE),
    (dict(ldx=68), SHAPE), (dict(add=A + 2), MISALIGNED), (dict(lda=60), SHAPE), (dict(total=A + 4), MISALIGNED), (dict(lds=56), SHAPE),
    (dict(out=A + 8), MISALIGNED), (dict(ldo=56), SHAPE), (dict(ldo=1 << 40), SHAPE), (dict(total=None, out=None), INVALID), (dict(total=4 * A), INVALID),
    (dict(total=A, lds=72), INVALID), (dict(total=2 * A, lds=72), INVALID), (dict(out=A, ldo=72), INVALID), (dict(out=A, xt=1, total=None), INVALID),
    (dict(total=2 * A, xt=1), INVALID)])
def test_norms_that_are_refused(lib, change, status):
    assert norm(lib, **change) == status


@pytest.mark.parametrize("change,status", [
    (dict(group=-1), SHAPE), (dict(group=4), SHAPE), (dict(group=24), SHAPE), (dict(group=1024), SHAPE), (dict(values=None), INVALID),
    (dict(scale=None), INVALID), (dict(values=5 * A + 8), MISALIGNED), (dict(scale=A + 2), MISALIGNED), (dict(ld=56), SHAPE), (dict(ld=68), SHAPE),
    (dict(ld_scale=3), SHAPE), (dict(values=A), INVALID), (dict(values=2 * A), INVALID), (dict(values=3 * A), INVALID), (dict(values=4 * A), INVALID)])
def test_rows_in_8_bits_that_are_refused(lib, change, status):
    assert norm(lib, r8=rows8(**change)) == status


def test_no_rows_are_done_at_once(lib):
    assert norm(lib, n=0) == OK and norm(lib, n=0, x=None) == OK
    assert lib.lora_add_norm(None, 0, A, 64, 0, None, 0, 0, A, 64, None, 0, None, None) == INVALID


def sample(lib, logits=A, ld=100, dtype=1, n=3, vocab=100, how=True, u=A, token=A, prob=A, **kw):
    d = dict(temperature=A, top_k=A, top_p=A, min_p=A)
    d.update(kw)
    return lib.lora_sample(logits, ld, dtype, n, vocab, C.byref(B._Sampling(**d)) if how else None, u, token, prob, None)


@pytest.mark.parametrize("change,status", [
    (dict(how=False), INVALID), (dict(dtype=2), INVALID), (dict(n=-1), INVALID), (dict(n=L.LORA_MAX_ROWS_LONG + 1), LARGE), (dict(vocab=0), SHAPE),
    (dict(ld=99), SHAPE), (dict(ld=1 << 40), SHAPE), (dict(vocab=L.LORA_SAMPLE_MAX_VOCAB + 1, ld=1 << 23), LARGE), (dict(logits=None), INVALID),
    (dict(u=None), INVALID), (dict(token=None), INVALID), (dict(logits=A + 2), MISALIGNED), (dict(logits=A + 1, dtype=0), MISALIGNED),
    (dict(u=A + 2), MISALIGNED), (dict(token=A + 1), MISALIGNED), (dict(prob=A + 2), MISALIGNED), (dict(temperature=A + 2), MISALIGNED),
    (dict(top_k=A + 2), MISALIGNED), (dict(top_p=A + 2), MISALIGNED), (dict(min_p=A + 2), MISALIGNED)])
def test_samplings_that_are_refused(lib, change, status):
    assert sample(lib, **change) == status


def test_no_rows_are_sampled_at_once(lib):
    assert sample(lib, n=0) == OK and sample(lib, n=0, logits=None, u=None, token=None) == OK


def test_handles_look_at_their_tensors():
    f, i = torch.zeros(8), torch.zeros(8, dtype=torch.int32)
    b = torch.zeros((4, 16), dtype=torch.uint8)
    for bad in (lambda: L.Norm(torch.zeros(8, dtype=torch.float16)), lambda: L.Norm(torch.zeros((2, 8))), lambda: L.Norm(torch.zeros(16)[::2]),
                lambda: L.Norm(f, width=16), lambda: L.Rows8(torch.zeros((4, 16)), torch.zeros((4, 1))), lambda: L.Rows8(b, torch.zeros((4, 2))),
                lambda: L.Rows8(b, torch.zeros((4, 1)), 8), lambda: L.Rows8(b, torch.zeros((3, 1))), lambda: L.Rows8(b.t(), torch.zeros((16, 1))),
                lambda: L.Rows8(b, torch.zeros((4, 1), dtype=torch.float64)), lambda: L.Sampling(temperature=i), lambda: L.Sampling(top_k=f),
                lambda: L.Sampling(top_p=f.double()), lambda: L.Sampling(min_p=f[::2])):
        with pytest.raises(ValueError):
            bad()
    x = torch.zeros((9, 16))
    for kw in (dict(n_rows=9, how=L.Sampling(temperature=f), u=torch.zeros(9), token=torch.zeros(9, dtype=torch.int32)),
               dict(n_rows=8, how=L.Sampling(), u=torch.zeros(7), token=i), dict(n_rows=8, how=L.Sampling(), u=f, token=f),
               dict(n_rows=8, how=L.Sampling(), u=f, token=i, prob=i)):
        with pytest.raises(ValueError):
            L.lora_sample(x, 16, vocab=16, stream=0, **kw)
    with pytest.raises(ValueError):
        L.lora_add_norm(L.Norm(width=16), 5, x, 16, None, 0, x, 16, None, 0, L.Rows8(b, torch.zeros((4, 1))), stream=0)
    with pytest.raises(ValueError):
        L.lora_add_norm(L.Norm(width=24), 4, x, 24, None, 0, x, 24, None, 0, L.Rows8(b, torch.zeros((4, 1))), stream=0)


def test_every_argument_arrives_where_ctypes_puts_it():
    b = [Buffer(1000 + i, 0x7F0000000000 + 4096 * i) for i in range(5)]
    a = [v.address for v in b]
    big = 1 << 35
    lib = L.load_library()
    names = ("lora_add_norm", "lora_sample")
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
    w, r8, how = (Holder(x()) for x in (B._Norm, B._Rows8, B._Sampling))
    r = lambda h: C.byref(h.c)                                                  # noqa: E731
    B._calls().bind_step(addresses)
    try:
        for short, long_way in [
            (lambda: L.lora_add_norm(w, 5, b[0], big, b[1], 16, b[2], 24, b[3], 32, r8, 1, 0, stream=9),
             lambda: through["lora_add_norm"](r(w), 5, a[0], big, 1, a[1], 16, 0, a[2], 24, a[3], 32, r(r8), 9)),
            (lambda: L.lora_add_norm(w, 5, b[0], 8, None, 0, None, 0, b[3], 32, add_dtype=1, stream=9),
             lambda: through["lora_add_norm"](r(w), 5, a[0], 8, 0, None, 0, 1, None, 0, a[3], 32, None, 9)),
            (lambda: L.lora_sample(b[0], big, 7, 100, how, b[1], b[2], b[3], dtype=0, stream=9),
             lambda: through["lora_sample"](a[0], big, 0, 7, 100, r(how), a[1], a[2], a[3], 9)),
            (lambda: L.lora_sample(b[0], 8, 7, 100, how, b[1], b[2], stream=9),
             lambda: through["lora_sample"](a[0], 8, 1, 7, 100, r(how), a[1], a[2], None, 9)),
        ]:
            short()
            assert long_way() == 0
            (name, got), (name2, want) = calls[-2:]
            assert name == name2 and got == want, name
    finally:
        B._calls().bind_step({n: C.cast(getattr(lib, n), C.c_void_p).value for n in names})
    with pytest.raises(L.LoraError):                  # converted, then refused for the empty structures
        L.lora_add_norm(w, 1, b[0], 8, None, 0, b[1], 8, None, 0, stream=0)
    with pytest.raises(AttributeError):
        L.lora_add_norm(b[0], 1, b[0], 8, None, 0, b[1], 8, None, 0, stream=0)
    with pytest.raises(OverflowError):
        L.lora_sample(b[0], 8, 1 << 40, 8, how, b[1], b[2], stream=0)
