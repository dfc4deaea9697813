"""lora_add_norm at the ends of its numbers: constants under the root that are as large as huge rows' squares."""
import numpy as np
import pytest
import torch

import paper_2604_07173_amd as L
from test_gpu_add_norm import call, check, formula

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("W", [8, 64, 136, 1024, 2056, 40000])
@pytest.mark.parametrize("scale,eps", [(3e19, 3e38), (3e19, 1e30), (6e18, 3.3e38), (1e17, 3.3e38), (1e30, 3e38), (1.0, 3.3e38), (6e18, 1e-5)])
def test_a_large_constant_under_the_root(W, scale, eps):
    """The sum of squares is infinite in 32 bits, or it is not and its mean with eps is, or neither."""
    g = torch.Generator().manual_seed(W)
    x = (scale * (0.5 + torch.rand((5, W), generator=g))).cuda()
    w = (0.5 + torch.rand(W, generator=g)).cuda()
    got = call(x, None, w, group=128, eps=eps)
    check(got, formula(x, None, w, float(np.float32(eps)), 0.0), 128)
