"""What the binding of the paged cache refuses before a call: tensors of another type or size than the device code reads and writes."""
import pytest
import torch

import paper_2604_07173_amd as L


def i32(*shape):
    return torch.zeros(shape, dtype=torch.int32)


def setup(n_pages=10, n_seqs=3):
    k = torch.zeros((1, n_pages, 2, 16, 8), dtype=torch.bfloat16)
    states = [L.KvState(i32(n_seqs, 4), i32(n_seqs), i32(n_pages)) for _ in range(2)]
    return L.KvCache(k, k.clone()), states[0], states[1], L.KvMoves(n_pages, n_seqs, device="cpu")


@pytest.mark.parametrize("bad", [
    torch.zeros(3, dtype=torch.int64), torch.zeros(3), torch.zeros(3, dtype=torch.int16), i32(2), i32(0), i32(6)[::2]])
@pytest.mark.parametrize("which", [0, 1])
def test_a_plan_of_other_types_and_sizes(bad, which):
    cache, state, to, moves = setup()
    args = [i32(3), i32(3)]
    args[which] = bad
    with pytest.raises(ValueError, match=("src", "new_len")[which]):
        L.lora_kv_plan(cache, state, to, *args, moves, stream=0)


@pytest.mark.parametrize("short", [0, 1])
@pytest.mark.parametrize("compact", [False, True])
def test_fewer_counts_than_the_cache_has_pages(short, compact):
    """page_ref is written (in `from`: read, where a plan is refused) for every page of the cache."""
    cache, state, to, moves = setup()
    states = [state, to]
    states[short] = L.KvState(i32(3, 4), i32(3), i32(9))
    with pytest.raises(ValueError, match="page_ref"):
        if compact:
            L.lora_kv_compact(cache, *states, moves, stream=0)
        else:
            L.lora_kv_plan(cache, *states, i32(3), i32(3), moves, stream=0)


def test_a_cache_of_another_16_bit_type():
    k = torch.zeros((1, 4, 2, 16, 8), dtype=torch.float16)
    for pair in ((k, k.clone()), (k.bfloat16(), k), (k, k.bfloat16())):
        with pytest.raises(ValueError, match="bf16"):
            L.KvCache(*pair)
    for kind in (torch.bfloat16, torch.int16):                 # the type, or its bits
        assert L.KvCache(k.to(kind), k.to(kind)).c.head_dim == 8


@pytest.mark.parametrize("bad", [torch.zeros(1), i32(0), torch.zeros(1, dtype=torch.int16), torch.zeros(4, dtype=torch.uint8)])
def test_a_status_of_another_type(bad):
    """The calls set bits of a 32-bit word there."""
    with pytest.raises(ValueError, match="status"):
        L.KvBatch(i32(4), i32(3), i32(3, 2), 3, status=bad)


@pytest.mark.parametrize("good", [i32(1), i32(), i32(5)[2:3], torch.zeros(1, dtype=torch.uint32)])
def test_a_status_word(good):
    assert L.KvBatch(i32(4), i32(3), i32(3, 2), 3, status=good).c.status == good.data_ptr()
