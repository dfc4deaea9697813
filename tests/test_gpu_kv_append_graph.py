"""lora_rope_append recorded in a graph: every replay writes the cache, which is put back in between."""
import torch

import pytest

import paper_2604_07173_amd as L
from kv_common import KvCase

pytestmark = pytest.mark.gpu


def test_every_replay_writes_the_cache():
    case = KvCase([1] * 20, list(range(30, 50)), dim=128, stale=0.0).device()
    x = torch.randn((20, 8 * 128), device="cuda").bfloat16()
    out = torch.zeros((20, 512), dtype=torch.bfloat16, device="cuda")
    rope = L.Rope(128)
    blank_k, blank_v = case.kd.clone(), case.vd.clone()
    call = lambda: L.lora_rope_append(case.cache, 0, case.batch, rope, x, 1024, x[:, 512:], 1024, x[:, 768:], 1024, out, 512, 4)  # noqa: E731

    def wipe():
        out.zero_(), case.kd.copy_(blank_k), case.vd.copy_(blank_v)

    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for _ in range(3):
        x.normal_()
        case.batch.seq_len.sub_(1)
        wipe()
        call()
        want = out.clone(), case.kd.clone(), case.vd.clone()
        assert not torch.equal(want[1], blank_k) and not torch.equal(want[2], blank_v)
        wipe()
        graph.replay()
        torch.cuda.synchronize()
        for got, w in zip((out, case.kd, case.vd), want):
            assert torch.equal(got, w)


def test_v_keeps_its_bits():
    """Every bf16 value that is a number or an infinity, subnormal ones among them, arrives as it is; NaN stays NaN."""
    bits = torch.arange(1 << 16, dtype=torch.int32).to(torch.int16)
    v = bits.view(torch.bfloat16).view(512, 128).cuda()
    case = KvCase([512], [512], 1, 1, 128, stale=0.0).device()
    L.lora_rope_append(case.cache, 0, case.batch, None, None, 0, v, 128, v, 128, None, 0, 0)
    torch.cuda.synchronize()
    for t in (case.kd, case.vd):
        got = t[0, torch.from_numpy(case.table[0].astype("int64")).cuda(), 0].reshape(512, 128)
        nan = torch.isnan(v)
        assert torch.equal(torch.isnan(got), nan)
        assert torch.equal(got.view(torch.int16)[~nan], v.view(torch.int16)[~nan])
