"""The paged cache's calls through the extension module: every argument arrives where ctypes puts it, and what
cannot be converted is refused."""
import contextlib
import ctypes as C

import pytest

import paper_2604_07173_amd as L
from paper_2604_07173_amd import binding as B

ENTRIES = ("lora_rope_append", "lora_kv_attention", "lora_kv_plan", "lora_kv_compact", "lora_kv_copy_pages")


class Buffer:
    """A tensor as the module sees one."""

    def __init__(self, n, address):
        self.n, self.address = n, address

    def data_ptr(self):
        return self.address

    def numel(self):
        return self.n

    def element_size(self):
        return 2


class Holder:
    def __init__(self, c):
        self.c = c


@contextlib.contextmanager
def recorded():
    lib = L.load_library()
    calls, keep, addresses, through_ctypes = [], [], {}, {}
    for name in ENTRIES:
        types = getattr(lib, name).argtypes

        def note(*args, name=name, types=types):
            calls.append((name, [C.addressof(v.contents) if v and issubclass(t, C._Pointer) else None if issubclass(t, C._Pointer) else v
                                 for t, v in zip(types, args)]))
            return 0

        proto = C.CFUNCTYPE(C.c_int, *types)
        keep.append(proto(note))
        addresses[name] = C.cast(keep[-1], C.c_void_p).value
        through_ctypes[name] = proto(addresses[name])
    B._calls().bind_kv(addresses)
    try:
        yield calls, through_ctypes
    finally:
        B._calls().bind_kv({n: C.cast(getattr(lib, n), C.c_void_p).value for n in ENTRIES})


def test_every_argument_arrives_where_ctypes_puts_it():
    b = [Buffer(1000 + i, 0x7F0000000000 + 4096 * i) for i in range(8)]
    a = [v.address for v in b]
    big = 1 << 40
    cache, batch, rope, state, to, moves = (Holder(t()) for t in (B._KvCache, B._KvBatch, B._Rope, B._KvState, B._KvState, B._KvMoves))
    r = lambda h: C.byref(h.c)                                                  # noqa: E731
    with recorded() as (calls, ct):
        pairs = [
            (lambda: L.lora_rope_append(cache, 2, batch, rope, b[0], big, b[1], 16, b[2], 24, b[3], 32, 40, L.LORA_DTYPE_F32, 9),
             lambda: ct["lora_rope_append"](r(cache), 2, r(batch), r(rope), a[0], big, a[1], 16, a[2], 24, a[3], 32, 40, 1, 9)),
            (lambda: L.lora_rope_append(cache, 0, batch, None, None, 0, b[1], 16, a[2], 24, None, 0, 0, stream=9),
             lambda: ct["lora_rope_append"](r(cache), 0, r(batch), None, None, 0, a[1], 16, a[2], 24, None, 0, 0, 0, 9)),
            (lambda: L.lora_kv_attention(cache, 3, batch, b[0], 8, 32, b[1], big, b[2], 0.125, b[3], causal=False, window=7, stream=9),
             lambda: ct["lora_kv_attention"](r(cache), 3, r(batch), a[0], 8, 32, a[1], big, a[2], 0.125, 0, 7, a[3], 2006, 9)),
            (lambda: L.lora_kv_plan(cache, state, to, b[0], b[1], moves, 9),
             lambda: ct["lora_kv_plan"](r(cache), r(state), r(to), a[0], a[1], r(moves), 9)),
            (lambda: L.lora_kv_compact(cache, state, to, moves, 9), lambda: ct["lora_kv_compact"](r(cache), r(state), r(to), r(moves), 9)),
            (lambda: L.lora_kv_copy_pages(cache, moves, 77, 9), lambda: ct["lora_kv_copy_pages"](r(cache), r(moves), 77, 9)),
        ]
        for short, long_way in pairs:
            short()
            assert long_way() == 0
            (name, got), (name2, want) = calls[-2:]
            assert name == name2 and got == want, name
        assert {name for name, _ in calls} == set(ENTRIES)


def test_what_cannot_be_converted_is_refused():
    cache, batch, x = Holder(B._KvCache()), Holder(B._KvBatch()), Buffer(64, 4096)

    def attend(c=cache, b=batch, layer=0, scale=1.0, ws=x, q=x):
        return L.lora_kv_attention(c, layer, b, q, 8, 1, x, 8, None, scale, ws, stream=0)

    with pytest.raises(L.LoraError):                  # converted, then refused for the empty cache
        attend()
    with pytest.raises(L.LoraError):
        attend(c=None)
    with pytest.raises(AttributeError):
        attend(c=x)
    with pytest.raises(TypeError):
        attend(b=Holder((C.c_char * 4)()))
    with pytest.raises(TypeError):
        attend(scale="1")
    with pytest.raises(OverflowError):
        attend(layer=1 << 40)
    with pytest.raises(AttributeError):
        attend(ws=None)
    with pytest.raises(AttributeError):
        attend(q=object())
