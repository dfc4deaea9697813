"""Values in e4m3 are the quotients of y and its scale, as fp32 has them, to the nearest: equal, at and beside the ties between two
values too, where a product with a rounded reciprocal comes out one step apart."""
import numpy as np
import pytest
import torch

from test_gpu_add_norm import call

pytestmark = pytest.mark.gpu


def near_ties(W, group, seed):
    """Weights that a row of ones leaves as they are, and most of which are halfway between two values of their group, or next to it."""
    rng = np.random.default_rng(seed)
    w = np.empty(W, np.float32)
    for at in range(0, W, group):
        n = min(group, W - at)
        most = np.float32(np.exp2(rng.uniform(-60, 60)) * rng.uniform(1, 2))
        scale = most / np.float32(448)
        steps = rng.integers(16, 32, n) + 0.5 * rng.integers(0, 2, n)          # five bits: a value of four, or a tie
        v = (steps / 16 * np.exp2(rng.integers(-6, 8, n)) * np.float64(scale)).astype(np.float32)
        v = np.where(rng.random(n) < 0.3, v, np.nextafter(v, np.float32(np.inf) * rng.choice([-1, 1], n).astype(np.float32)))
        v = np.minimum(v, most) * rng.choice([-1, 1], n)
        v[rng.integers(n)] = most
        w[at:at + n] = v
    return torch.from_numpy(w)


@pytest.mark.parametrize("W,group", [(64, 8), (1000, 64), (4096, 128), (5000, 512), (2056, 0), (40000, 128)])
def test_quotients_are_rounded_to_the_nearest(W, group):
    for seed in range(6):
        w = near_ties(W, group or W, seed)
        x = torch.ones(3, W)
        x[1] = -1
        # the mean of the squares is one, and what eps adds is lost: y is the weight itself
        _, _, y8, scale = call(x.cuda(), None, w.cuda(), group=group, eps=1e-37)
        g = group or W
        top = torch.nn.functional.pad(w, (0, -W % g)).view(-1, g).abs().amax(1)
        want_scale = top / 448.0
        assert torch.equal(scale.cpu(), want_scale.expand(3, -1))
        want = (w / want_scale.repeat_interleave(g)[:W]).clamp(-448, 448).to(torch.float8_e4m3fn).float()
        assert torch.equal(y8.float().cpu(), torch.stack([want, -want, want]))


def test_the_smallest_and_the_largest():
    """Scales down to 2^-126, and groups whose largest value is infinite: zeros beside it."""
    w = torch.cat([2.0 ** -117 * torch.tensor([1.0, 0.3, -0.51, 1e-3, 0.0, 0.77, -0.124, 0.9]), 1e-20 * torch.rand(8), 3e38 * torch.rand(8), torch.zeros(8)])
    _, _, y8, scale = call(torch.ones(2, 32).cuda(), None, w.cuda(), group=8, eps=1e-37)
    top = w.view(4, 8).abs().amax(1)
    want_scale = torch.where(top == 0, 1.0, top / 448.0)
    assert torch.equal(scale.cpu(), want_scale.expand(2, -1))
    want = (w / want_scale.repeat_interleave(8)).clamp(-448, 448).to(torch.float8_e4m3fn).float()
    assert torch.equal(y8.float().cpu(), want.expand(2, -1))
    w = torch.tensor([1.0, 3e38, 2.0, 0.0, 0.0, 5.0, 7.0, 1.0])
    x = torch.tensor([[1.0, 2.0, 1.0, 1.0, 1.0, 1.0, 1.0, 1.0]])
    _, _, y8, scale = call(x.cuda(), None, w.cuda(), group=8)
    assert scale[0, 0] == float("inf")
    assert torch.isnan(y8[0, 1].float()) and (y8[0, [0, 2, 3, 4, 5, 6, 7]].float() == 0).all()
