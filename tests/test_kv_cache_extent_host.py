"""Layouts of caches that the calls take and refuse, and caches whose last element lies further out than 64 bits of elements can say, which
are refused however the strides wrap."""
import ctypes as C
import itertools

import pytest

import paper_2604_07173_amd as L
from paper_2604_07173_amd import binding as B

A = 0x10000
OK, SHAPE, LARGE = 0, -2, -8


def status(**kw):
    d = dict(k=A, v=A, n_layers=2, n_pages=10, n_heads=4, page_size=16, head_dim=64, layer_stride=40960, page_stride=4096,
             head_stride=1024, token_stride=64)
    d.update(kw)
    return L.load_library().lora_kv_copy_pages(C.byref(B._KvCache(**d)), C.byref(B._KvMoves(1, 0, A, A, A, A, 1 << 20)), 0, None)


@pytest.mark.parametrize("change", [
    dict(n_pages=(1 << 16) + 1, page_stride=1 << 48),                        # 2^64: wraps to the page alone
    dict(n_pages=(1 << 20) + 1, page_stride=1 << 44),
    dict(n_pages=(1 << 30) + 5, page_stride=1 << 40, layer_stride=1 << 44),
    dict(n_heads=32767, head_stride=1 << 48, page_stride=1 << 48, n_pages=1),
    dict(n_layers=16384, layer_stride=1 << 48),                              # elements fit, bytes do not
    dict(n_pages=1 << 20, page_stride=1 << 42, n_layers=1),
])
def test_extents_that_do_not_fit(change):
    assert status(**change) == LARGE


def test_large_extents_that_fit():
    assert status() == OK
    assert status(n_pages=1 << 24, page_stride=1 << 20, layer_stride=1 << 45) == OK
    assert status(n_layers=256, layer_stride=1 << 48) == OK
    assert status(n_pages=(1 << 31) - 1024, n_layers=1) == OK


DIMS = dict(l=("n_layers", "layer_stride", 2), p=("n_pages", "page_stride", 10), h=("n_heads", "head_stride", 4),
            t=("page_size", "token_stride", 16))


@pytest.mark.parametrize("order", list(itertools.permutations("lpht")), ids="".join)
def test_every_order_is_taken_and_none_that_overlaps(order):
    strides, each = {}, 64
    for d in reversed(order):
        strides[DIMS[d][1]] = each
        each *= DIMS[d][2]
    assert status(**strides) == OK
    for d in order:                                # a stride eight less: one thing begins inside another one
        assert status(**dict(strides, **{DIMS[d][1]: strides[DIMS[d][1]] - 8})) == SHAPE
        assert status(**dict(strides, **{DIMS[d][0]: 1, DIMS[d][1]: 0})) == OK       # of which there is one: any stride


@pytest.mark.parametrize("n_pages", [(1 << 31) - 1023, (1 << 31) - 512, (1 << 31) - 1])
def test_more_pages_than_the_lists_can_number(n_pages):
    """Lists are made in chunks of 1024 pages, numbered in 32 bits: the last chunk has to end below 2^31."""
    assert status(n_pages=n_pages, n_layers=1) == LARGE
    assert L.lora_kv_moves_ws_bytes(n_pages, 4) == 0
    assert L.lora_kv_moves_ws_bytes((1 << 31) - 1024, 4) > 16 << 31
