"""lora_sample against its definition in 64 bits: the same tokens wherever no border is within the weights' last bits."""
import math

import numpy as np
import pytest
import torch

import paper_2604_07173_amd as L
from sample_common import one_row

pytestmark = pytest.mark.gpu


def call(x, T=None, k=None, p=None, least=None, u=None, stream=None, prob=True, vocab=None):
    R = x.shape[0]
    V = vocab or x.shape[1]
    dev = lambda v, t: None if v is None else torch.from_numpy(np.broadcast_to(np.asarray(v, t), (R,)).copy()).cuda()      # noqa: E731
    how = L.Sampling(dev(T, np.float32), dev(k, np.int32), dev(p, np.float32), dev(least, np.float32))
    token = torch.full((R,), -9, dtype=torch.int32, device="cuda")
    pr = torch.full((R,), -9.0, device="cuda") if prob else None
    ld = x.stride(0) if R > 1 else x.shape[1]
    L.lora_sample(x, ld, R, V, how, dev(u, np.float32), token, pr, dtype=L.LORA_DTYPE_F32 if x.dtype == torch.float32 else L.LORA_DTYPE_BF16, stream=stream)
    return token, pr


def check(x, T=None, k=None, p=None, least=None, u=None, most_unsure=0.02):
    """x: on the device."""
    R = x.shape[0]
    token, prob = (t.cpu() for t in call(x, T, k, p, least, u))
    host = x.double().cpu().numpy()
    at = lambda v, r, none: none if v is None else float(np.broadcast_to(np.float32(v), (R,))[r])                         # noqa: E731
    unsure = 0
    for r in range(R):
        want, wp, others = one_row(host[r], at(T, r, 1.0), int(at(k, r, 0)), at(p, r, 1.0), at(least, r, 0.0), at(u, r, 0.0))
        if others is not None:
            unsure += 1
            assert int(token[r]) in others, (r, int(token[r]), others[:9])
            continue
        assert int(token[r]) == want, (r, int(token[r]), want)
        # the sum of V weights, each off by half a step, and three roundings to 32 bits
        assert abs(float(prob[r]) - wp) <= wp * (2.0 ** -22 + x.shape[1] * 2.0 ** -39), (r, float(prob[r]), wp)
    assert unsure <= most_unsure * R + 1
    return token


def logits(R, V, kind=torch.float32, seed=0, scale=2.5, pad=0):
    g = torch.Generator().manual_seed(seed + V)
    x = scale * torch.randn((R, V + pad), generator=g)
    likely = torch.randint(0, V, (R, 12), generator=g)
    x.scatter_add_(1, likely, 10.0 * torch.rand((R, 12), generator=g))
    return x.to(kind).cuda()[:, :V]


def us(R, seed=0):
    return np.random.default_rng(seed).random(R).astype(np.float32)


RULES = [dict(), dict(T=0.7), dict(T=1.5, k=50), dict(p=0.9), dict(T=0.8, k=40, p=0.95), dict(least=0.05), dict(T=1.2, k=300, p=0.8, least=0.01), dict(T=0.0),
         dict(k=1), dict(p=0.0), dict(p=1e-6), dict(least=1.0)]


@pytest.mark.parametrize("V", [1, 2, 7, 63, 257, 1024, 4099, 8192, 8193, 32000, 50257, 131072])
@pytest.mark.parametrize("kind", [torch.float32, torch.bfloat16])
def test_rules(V, kind):
    R = 12 if V < 20000 else 5
    for i, rule in enumerate(RULES):
        check(logits(R, V, kind, seed=i), u=us(R, i), **rule)


@pytest.mark.parametrize("V", [1 << 20, (1 << 22) - 3])
def test_large_vocabularies(V):
    # With 2^22 tokens a weight is a multiple of 2^-40, so sums may be off by 2^22 * 2^-41 = 2^-19, and the edges between tokens, of
    # weights from 2^-40 on, lie closer than that: the oracle's list of tokens is all that can be asked for there
    for rule in (dict(), dict(T=2.0, k=1000, p=0.9), dict(p=0.99)):
        check(logits(2, V, seed=5), u=us(2, V), most_unsure=1.0, **rule)


@pytest.mark.parametrize("kind", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("levels", [1, 2, 5, 40])
def test_equal_logits(kind, levels):
    """Whole weights in places with few values: borders lie among equal tokens, the lowest numbers are kept."""
    V, R = 5000, 40
    g = torch.Generator().manual_seed(levels)
    x = torch.randint(0, levels, (R, V), generator=g).to(kind).cuda()
    for k, p in ((0, 1.0), (1, 1.0), (37, 1.0), (V - 1, 1.0), (0, 0.3), (1234, 0.77)):
        check(x, u=us(R, k), k=k, p=p, most_unsure=0.1)
    token = call(x, k=1, u=us(R))[0].cpu()
    assert torch.equal(token.long(), torch.from_numpy(np.argmax(x.float().cpu().numpy(), 1)))


@pytest.mark.parametrize("spread", [1e-6, 1e-4, 3e-2])
def test_many_values_in_one_bin(spread):
    """More values in a bin of weights than a workgroup keeps: they are looked through again for every step."""
    V = 60000
    g = torch.Generator().manual_seed(1)
    for offset in (0.0, 11.0):                       # around zero keys of both signs, elsewhere a few hundred steps of a float
        x = (offset + spread * torch.randn((4, V), generator=g)).cuda()
        check(x, u=us(4), k=20000)
        check(x, u=us(4, 1), p=0.4)
        check(x, u=us(4, 2), k=30000, p=0.5)


def test_every_row_has_its_own_rule():
    rng = np.random.default_rng(4)
    R, V = 200, 3001
    x = logits(R, V)
    check(x, T=rng.choice([0.0, 0.3, 1.0, 2.0], R), k=rng.choice([0, 1, 5, 100, 3000, 3001, 9999], R), p=rng.choice([0.1, 0.5, 0.9, 0.999, 1.0, 2.0], R),
          least=rng.choice([0.0, 0.01, 0.3], R), u=us(R, 9))


@pytest.mark.parametrize("V,k", [(5000, 65), (5000, 190), (20000, 257), (20000, 600), (20000, 768), (20000, 769), (60000, 4000)])
@pytest.mark.parametrize("kind", [torch.float32, torch.bfloat16])
def test_lists_of_all_lengths(V, k, kind):
    """Lists that are compared in pairs, counted in bins, and none at all, with every other limit on top."""
    for i, rule in enumerate((dict(), dict(p=0.7), dict(p=0.999), dict(least=0.02), dict(p=0.9, least=0.001, T=1.4), dict(T=0.4, p=0.5), dict(T=30.0, p=0.9))):
        check(logits(6, V, kind, seed=i), u=us(6, i), k=k, **rule)
    x = logits(6, V, kind)
    x[:, : V // 3] = 4.0                              # equal ones, more than a list takes
    check(x, u=us(6), k=k, p=0.8)


@pytest.mark.parametrize("V,R", [(1500, 6), (12000, 6), (12000, 260), (50257, 4), (200001, 4)])
@pytest.mark.parametrize("left", [1, 2, 40, 129, 300, 700, 5000, 20000])
def test_rows_of_which_a_mask_leaves_few(V, R, left):
    """Fewer tokens than top_k, than the workgroup has threads, than a list takes, in a stretch of the row and anywhere in it."""
    g = torch.Generator().manual_seed(left)
    left = min(left, V)
    for near in (False, True):
        x = torch.full((R, V), -math.inf)
        for r in range(R):
            at = torch.randperm(V, generator=g)[:left] if not near else (torch.arange(left) + int(torch.randint(0, V, (1,), generator=g))) % V
            x[r, at] = 2.5 * torch.randn(left, generator=g)
        x = x[:6].cuda() if R <= 6 else x.cuda()
        rows = np.arange(R) % 4
        check(x, k=np.array([1, 50, 400, 760])[rows], u=us(R))
        check(x, k=np.array([50, 400, 760, 3000])[rows], p=0.9, u=us(R, 1), T=1.3)
        if R > 6:
            return


def test_logits_as_far_apart_as_floats_are():
    """Differences that are infinite in 32 bits."""
    x = torch.full((4, 3000), -math.inf)
    x[:, 1234] = 3e38
    x[:, 77] = -3e38
    x[2:, 78] = 1e38
    x = x.cuda()
    for k in (1, 2, 3, 50):
        check(x, T=2e38, k=k, u=us(4, k))
        check(x, T=2e38, k=k, p=0.97, u=us(4, k))


def test_all_of_u():
    """One row's tokens over a fine grid of u, the ends among it."""
    R = 500
    x = logits(1, 700).repeat(R, 1)
    u = np.linspace(0, 1, R, dtype=np.float32)
    check(x, u=u, T=0.9, k=60, p=0.97)
    token = call(x, u=u)[0]
    assert (token[1:] >= token[:-1]).all()


@pytest.mark.parametrize("u", [float("nan"), -3.0, -0.0, 1.0, 7.0, float("inf")])
def test_u_outside_its_range(u):
    check(logits(6, 900), u=np.full(6, u, np.float32), k=30)


@pytest.mark.parametrize("T", [float("nan"), -1.0, float("inf"), 1e-38, 1e-45, 1e30, 1e-3])
def test_temperatures_at_the_ends(T):
    check(logits(8, 1000), T=T, u=us(8), k=200)


@pytest.mark.parametrize("rule", [dict(p=float("nan")), dict(least=float("nan")), dict(p=-1.0), dict(least=-1.0), dict(least=5.0), dict(k=-3)])
def test_limits_that_are_none(rule):
    check(logits(8, 1000), u=us(8), **rule)


def test_masked_logits():
    inf, nan = float("inf"), float("nan")
    V = 2000
    x = logits(9, V).clone()
    x[0] = -inf                                      # nothing left
    x[1] = -inf
    x[1, 1234] = -50.0                               # one token
    x[2] = nan
    x[3, ::2] = nan
    x[4, 100:] = -inf
    x[5, [3, 77, 1999]] = inf                        # of these one
    x[6] = torch.finfo(torch.float32).min
    x[7, :] = torch.finfo(torch.float32).min
    x[7, 9] = 0.0
    x[8, 5] = torch.finfo(torch.float32).max
    for rule in (dict(), dict(k=10), dict(p=0.5), dict(T=0.0), dict(k=5, p=0.9, least=0.1, T=0.5)):
        token = check(x, u=us(9), **rule)
        assert token[0] == -1 and token[1] == 1234 and token[2] == -1 and token[5] in (3, 77, 1999) and token[7] == 9 and token[8] == 5


def test_zeros_of_both_signs_are_equal():
    x = torch.full((20, 600), -5.0)
    x[:, 100:300] = 0.0
    x[:, 100:300:2] = -0.0
    token = check(x.cuda(), u=us(20), k=50)
    assert (token >= 100).all() and (token < 150).all()


@pytest.mark.parametrize("kind,pad,start", [(torch.float32, 0, 1), (torch.float32, 3, 2), (torch.bfloat16, 0, 1), (torch.bfloat16, 5, 3)])
def test_rows_that_are_aligned_to_a_logit_only(kind, pad, start):
    """Odd strides and beginnings; columns behind the vocabulary would win."""
    V, R = 4097, 7
    wide = torch.full((R, V + pad + start), 60.0, dtype=kind, device="cuda")
    wide[:, start:start + V] = logits(R, V, kind)
    view = wide[:, start:start + V]
    for rule in (dict(), dict(T=0.8, k=40, p=0.9), dict(T=0.0)):
        check(view, u=us(R), **rule)


def test_settings_that_are_left_out_and_no_probabilities():
    x = logits(5, 3000)
    u = us(5)
    token, prob = call(x, u=u)
    assert torch.equal(call(x, T=1.0, k=0, p=1.0, least=0.0, u=u)[0], token)
    assert torch.equal(call(x, u=u, prob=False)[0], token)
    check(x, u=u)


def test_repeats_streams_and_graphs():
    R, V = 30, 32000
    x, u = logits(R, V), us(R)
    want = call(x, T=0.9, k=500, p=0.9, u=u)
    for _ in range(3):
        again = call(x, T=0.9, k=500, p=0.9, u=u)
        assert torch.equal(again[0], want[0]) and torch.equal(again[1], want[1])
    T, k, p, ud = torch.full((R,), 0.9, device="cuda"), torch.full((R,), 500, dtype=torch.int32, device="cuda"), torch.full((R,), 0.9, device="cuda"), torch.from_numpy(u).cuda()
    how, token, prob = L.Sampling(T, k, p), torch.zeros(R, dtype=torch.int32, device="cuda"), torch.zeros(R, device="cuda")
    L.lora_sample(x, V, R, V, how, ud, token, prob)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        L.lora_sample(x, V, R, V, how, ud, token, prob)
    for i in range(3):
        ud.copy_(torch.from_numpy(us(R, i)))
        token.fill_(-3)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(token, call(x, T=0.9, k=500, p=0.9, u=us(R, i))[0])
    token.fill_(-3)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    L.lora_sample(x, V, R, V, how, ud, token, prob, stream=side)
    side.synchronize()
    assert torch.equal(token, call(x, T=0.9, k=500, p=0.9, u=us(R, 2))[0])


@pytest.mark.parametrize("kind", [torch.float32, torch.bfloat16])
def test_many_rows_of_a_large_vocabulary(kind):
    """Rows that share CUs: lists of a quarter of the row and more, whole or of one bin."""
    R, V = 300, 20011
    rng = np.random.default_rng(8)
    check(logits(R, V, kind), T=rng.choice([0.0, 0.5, 1.0, 3.0], R), k=rng.choice([0, 40, 380, 400, 2000, 4900, 5100, 15000], R),
          p=rng.choice([0.5, 0.95, 1.0], R), least=rng.choice([0.0, 0.0, 0.01], R), u=us(R, 3))


def test_two_calls_at_once_on_two_streams():
    xs = [logits(70, 40000), logits(300, 9000, torch.bfloat16)]
    want = [call(x, T=0.8, k=3000, p=0.9, u=us(x.shape[0], 5)) for x in xs]
    streams = [torch.cuda.Stream() for _ in xs]
    torch.cuda.synchronize()
    for _ in range(5):
        got = []
        for x, st in zip(xs, streams):
            with torch.cuda.stream(st):              # what the call is given is written on its stream
                got.append(call(x, T=0.8, k=3000, p=0.9, u=us(x.shape[0], 5), stream=st))
        torch.cuda.synchronize()
        for g, w in zip(got, want):
            assert torch.equal(g[0], w[0]) and torch.equal(g[1], w[1])
