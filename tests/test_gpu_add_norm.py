"""lora_add_norm against its formula in 64 bits.

Bounds, in relative terms: the sum is one fp32 addition (2^-24) and its rounding (bf16: half a step, 2^-8).  y: a thread adds up at most
64 squares and twelve levels of a tree follow, each addition off by 2^-24 of it, half of which shows in the root; with the squares,
mean, root, division, weight and two products below 60 * 2^-24 < 2^-18, then bf16's 2^-8.  A scale is a maximum of such y.  e4m3: half a step is 2^-4 of a
value, 2^-10 where values are below 2^-6, of the scaled value."""
import math

import pytest
import torch

import paper_2604_07173_amd as L

pytestmark = pytest.mark.gpu

FP32 = 2.0 ** -18
BF16 = 2.0 ** -8 + FP32


def formula(x, add, w, eps, shift):
    s = x.double().cpu() + (0.0 if add is None else add.double().cpu())
    gain = (1.0 if w is None else w.double().cpu()) + shift
    return s, s / (s.square().mean(-1, keepdim=True) + eps).sqrt() * gain


def call(x, add, w, group=None, eps=1e-5, shift=0.0, total=True, out=True, total_to=None, out_to=None, stream=None):
    R, W = x.shape
    kind = lambda t: L.LORA_DTYPE_F32 if t is not None and t.dtype == torch.float32 else L.LORA_DTYPE_BF16        # noqa: E731
    ld = lambda t: 0 if t is None else t.stride(0) if R > 1 else t.shape[1]                                       # noqa: E731
    s = total_to if total_to is not None else torch.full((R, W), 7.0, dtype=x.dtype, device="cuda") if total else None
    y = out_to if out_to is not None else torch.full((R, W), 7.0, dtype=torch.bfloat16, device="cuda") if out else None
    y8 = scale = r8 = None
    if group is not None:
        y8 = torch.full((R, W), 1.0, device="cuda").to(torch.float8_e4m3fn)
        scale = torch.full((R, -(-W // group) if group else 1), 7.0, device="cuda")
        r8 = L.Rows8(y8, scale, group)
    norm = L.Norm(w, eps, shift, None if w is not None else W)
    L.lora_add_norm(norm, R, x, ld(x), add, ld(add), s, ld(s), y, ld(y), r8, kind(x), kind(add), stream=stream)
    return s, y, y8, scale


def check(got, want, group=None):
    (s, y, y8, scale), (ws, wy) = got, want
    if s is not None:
        assert ((s.double().cpu() - ws).abs() <= ws.abs() * (2.0 ** -24 if s.dtype == torch.float32 else 2.0 ** -8 + 2.0 ** -24)).all()
    if y is not None:
        err = (y.double().cpu() - wy).abs()
        assert (err <= wy.abs() * BF16 + 1e-38).all(), float((err / (wy.abs() * BF16 + 1e-38)).max())
    if y8 is not None:
        R, W = wy.shape
        g = group or W
        padded = torch.nn.functional.pad(wy, (0, -W % g)).view(R, -1, g)
        top = padded.abs().amax(-1)
        sc = torch.where(top == 0, torch.ones_like(top), top / 448.0)
        assert ((scale.double().cpu() - sc).abs() <= sc * FP32).all()
        per = scale.double().cpu().repeat_interleave(g, 1)[:, :W]
        err = (y8.double().cpu() * per - wy).abs()
        bound = wy.abs() * (2.0 ** -4 + 2 * FP32) + per * (2.0 ** -10 + FP32)
        assert (err <= bound).all(), float((err / bound).max())


def make(R, W, f32=False, add="bf16", seed=0, scale=3.0):
    g = torch.Generator().manual_seed(seed + R * 7 + W)
    t = lambda kind, f: (f * torch.randn((R, W), generator=g)).to(kind).cuda()                                    # noqa: E731
    x = t(torch.float32 if f32 else torch.bfloat16, scale)
    a = None if add is None else t(torch.float32 if add == "f32" else torch.bfloat16, 1.0)
    w = (1.0 + 0.3 * torch.randn(W, generator=g)).to(torch.bfloat16).cuda()
    return x, a, w


@pytest.mark.parametrize("W", [8, 16, 72, 504, 512, 520, 1024, 2048, 2056, 4096, 4104, 8192, 16376, 16384, 16392, 32768, 32776, 65536])
@pytest.mark.parametrize("R", [1, 5])
def test_widths(R, W):
    """Every number of threads and vectors per row, just full and just over."""
    x, a, w = make(R, W)
    check(call(x, a, w, group=128), formula(x, a, w, 1e-5, 0.0), 128)


@pytest.mark.parametrize("f32", [False, True])
@pytest.mark.parametrize("add", [None, "bf16", "f32"])
@pytest.mark.parametrize("wtype", [None, torch.bfloat16, torch.float32])
def test_types(f32, add, wtype):
    x, a, w = make(33, 1000, f32, add)
    w = None if wtype is None else w.to(wtype)
    check(call(x, a, w, group=0, shift=1.0, eps=1e-6), formula(x, a, w, 1e-6, 1.0), 0)


@pytest.mark.parametrize("group", [0, 8, 16, 32, 64, 128, 256, 512])
@pytest.mark.parametrize("W", [24, 1000, 4096, 5000])
def test_groups_of_columns_with_a_scale(group, W):
    x, a, w = make(9, W)
    x[:, :16] = 0
    a[:, :16] = 0                                    # a group of zeros has the scale 1
    x[3], a[3] = 0, 0
    got = call(x, a, w, group=group)
    check(got, formula(x, a, w, 1e-5, 0.0), group)
    assert (got[3][3] == 1.0).all() and (got[2][3].float() == 0).all()


@pytest.mark.parametrize("total,out,group", [(True, False, None), (False, True, None), (False, False, 64), (True, False, 64), (True, True, None)])
def test_what_is_not_wanted_may_be_left_out(total, out, group):
    x, a, w = make(70, 640)
    check(call(x, a, w, group=group, total=total, out=out), formula(x, a, w, 1e-5, 0.0), group)


@pytest.mark.parametrize("R", [3, 1000, 70001])
def test_many_rows_and_strides(R):
    """Columns of wider buffers; columns behind the rows stay; more rows than workgroups."""
    g = torch.Generator(device="cuda").manual_seed(R)
    wide = torch.randn((R, 3 * 64 + 8), generator=g, device="cuda").to(torch.bfloat16)
    x, a = wide[:, :64], wide[:, 72:136]
    sums, outs = (torch.full((R, 80), 5.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    w = torch.randn(64, generator=g, device="cuda")
    got = call(x, a, w, total_to=sums[:, 8:72], out_to=outs[:, 16:])
    check(got, formula(x, a, w, 1e-5, 0.0))
    assert (sums[:, :8] == 5).all() and (sums[:, 72:] == 5).all() and (outs[:, :16] == 5).all()


@pytest.mark.parametrize("W", [256, 4096, 40000])
def test_in_place(W):
    x, a, w = make(20, W)
    want = formula(x, a, w, 1e-5, 0.0)
    got = call(x, a, w, total_to=x, out_to=a)        # the sum takes x's place, the norm add's
    assert got[0] is x and got[1] is a
    check(got, want)
    x, a, w = make(20, W, seed=1)
    want = formula(x, a, w, 1e-5, 0.0)
    check(call(x, a, w, total=False, out_to=x), want)


@pytest.mark.parametrize("W", [8, 56, 64, 72, 128, 136, 256, 264])
@pytest.mark.parametrize("R", [1, 7, 33, 1001])
def test_rows_that_share_a_wave(R, W):
    """Each by itself, one that is scaled and one that is no number among them."""
    for group in (None, 0, 8, 64, 512):
        x, a, w = make(R, W, f32=True, add="f32")
        if R > 1:
            x[R // 2] *= 1e25
            a[R // 2] *= 1e25
            x[R // 3, 5] = math.nan
        good = torch.ones(R, dtype=torch.bool)
        good[R // 3] = R == 1
        s, y, y8, scale = call(x, a, w, group)
        ws, wy = formula(x, a, w, 1e-5, 0.0)
        pick = lambda v: None if v is None else v[good.to(v.device)]                        # noqa: E731
        check((pick(s), pick(y), pick(y8), pick(scale)), (pick(ws), pick(wy)), group)
        assert y[~good.cuda()].isnan().all()


def test_results_do_not_depend_on_other_rows_and_repeat():
    x, a, w = make(300, 4096)
    s, y, y8, scale = call(x, a, w, group=128)
    for _ in range(2):
        again = call(x, a, w, group=128)
        assert torch.equal(again[1], y) and torch.equal(again[2].view(torch.uint8), y8.view(torch.uint8)) and torch.equal(again[3], scale)
    one = call(x[77:78], a[77:78], w, group=128)
    assert torch.equal(one[1], y[77:78]) and torch.equal(one[3], scale[77:78])


@pytest.mark.parametrize("f32,scale", [(True, 1e25), (True, 1e38), (False, 1e30), (True, 1e-25), (False, 1e-20), (True, 1e-38)])
def test_huge_and_tiny_rows(f32, scale):
    """Squares beyond fp32 on either side; 1e38 times a normal number stays below fp32's largest only within three deviations."""
    g = torch.Generator().manual_seed(3)
    x = (scale * torch.rand((6, 768), generator=g)).to(torch.float32 if f32 else torch.bfloat16).cuda()
    w = torch.rand(768, generator=g).cuda()
    got = call(x, None, w)
    want = formula(x, None, w, 1e-5, 0.0)
    err = (got[1].double().cpu() - want[1]).abs()
    # where fp32 itself has fewer bits, below 2^-126: half its smallest step
    assert (err <= want[1].abs() * BF16 + 2.0 ** -126).all()


def test_numbers_that_are_none():
    x, _, w = make(4, 1024)
    x[1, 5], x[2, 700] = float("nan"), float("inf")
    s, y, y8, scale = call(x, None, w, group=128)
    clean = call(x[[0, 3]].contiguous(), None, w, group=128)
    assert torch.equal(y[[0, 3]], clean[1]) and torch.equal(scale[[0, 3]], clean[3])
    assert torch.isnan(y[1]).all() and torch.isnan(scale[1]).all() and torch.isnan(y8[1].float()).all()
    assert torch.isnan(y[2, 700]) and (y[2, :700] == 0).all() and (y[2, 701:] == 0).all()
    assert torch.isnan(scale[2, 5]) and torch.isnan(y8[2, 640:768].float()).all()
    assert (scale[2, :5] == 1).all() and (y8[2, :640].float() == 0).all()


def test_the_largest_value_is_reached_and_not_passed():
    x = torch.linspace(-1, 1, 4096).repeat(50, 1).mul(torch.rand(50, 1) * 1000).cuda()
    _, _, y8, scale = call(x, None, None, group=0)
    assert torch.isfinite(y8.float()).all() and (y8.float().abs().amax(1) == 448).all()


def test_in_a_graph_and_on_another_stream():
    x, a, w = make(64, 4096)
    want = call(x, a, w, group=128)
    s, y = torch.empty_like(x), torch.empty_like(x)
    y8, scale = torch.empty((64, 4096), dtype=torch.float8_e4m3fn, device="cuda"), torch.empty((64, 32), device="cuda")
    norm, r8 = L.Norm(w), L.Rows8(y8, scale, 128)
    run = lambda stream=None: L.lora_add_norm(norm, 64, x, 4096, a, 4096, s, 4096, y, 4096, r8, stream=stream)        # noqa: E731
    run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for _ in range(3):
        s.zero_(), y.zero_(), scale.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(s, want[0]) and torch.equal(y, want[1]) and torch.equal(scale, want[3])
    s.zero_(), y.zero_()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    run(side)
    side.synchronize()
    assert torch.equal(s, want[0]) and torch.equal(y, want[1])
