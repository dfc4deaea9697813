"""The types of the large tensors of a step's calls, without a GPU: a tensor of another type than the call is told would be read to another
length than it has."""
import pytest
import torch

import paper_2604_07173_amd as L

F32, BF16 = L.LORA_DTYPE_F32, L.LORA_DTYPE_BF16
f, b, h = (torch.zeros((4, 16), dtype=t) for t in (torch.float32, torch.bfloat16, torch.float16))


@pytest.mark.parametrize("logits,kw", [(b, {}), (b, dict(dtype=F32)), (f, dict(dtype=BF16)), (h, {}), (h, dict(dtype=BF16)), (f.double(), {}), (f.int(), {})])
def test_logits(logits, kw):
    with pytest.raises(ValueError, match="logits"):
        L.lora_sample(logits, 16, 4, 16, L.Sampling(), torch.zeros(4), torch.zeros(4, dtype=torch.int32), stream=0, **kw)


@pytest.mark.parametrize("x,add,total,out,kw,what", [
    (f, None, None, b, {}, "x"), (b, f, None, b, {}, "add"), (f, b, f, b, dict(add_dtype=F32), "x"), (f, b, f, b, dict(x_dtype=F32, add_dtype=F32), "add"),
    (b, b, f, b, {}, "total"), (f, f, b, b, dict(x_dtype=F32, add_dtype=F32), "total"), (b, b, b, f, {}, "out"), (h, None, None, b, {}, "x"),
    (b, b, None, h, {}, "out")])
def test_rows_of_a_norm(x, add, total, out, kw, what):
    with pytest.raises(ValueError, match=what):
        L.lora_add_norm(L.Norm(width=16), 4, x, 16, add, 16, total, 16, out, 16, stream=0, **kw)


def test_what_agrees_is_taken():
    """No rows: done at once, after all checks."""
    u, token = torch.zeros(4), torch.zeros(4, dtype=torch.int32)
    L.lora_sample(f, 16, 0, 16, L.Sampling(), u, token, stream=0)
    L.lora_sample(b, 16, 0, 16, L.Sampling(), u, token, dtype=BF16, stream=0)
    L.lora_sample(f.data_ptr(), 16, 0, 16, L.Sampling(), u, token, dtype=BF16, stream=0)       # an address has no type
    L.lora_add_norm(L.Norm(width=16), 0, b, 16, b, 16, b, 16, b, 16, stream=0)
    L.lora_add_norm(L.Norm(width=16), 0, f, 16, b, 16, f, 16, b, 16, x_dtype=F32, stream=0)
    L.lora_add_norm(L.Norm(width=16), 0, b, 16, f, 16, b, 16, None, 0, add_dtype=F32, stream=0)
    with pytest.raises(L.LoraError):
        L.lora_sample(f, 16, 0, 16, L.Sampling(), u, token, dtype=7, stream=0)
