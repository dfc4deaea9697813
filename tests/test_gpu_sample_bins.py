"""Sampling where the temperature puts all tokens in one bin, and so in the kernel's list: rows among memory whose values would win if they
were read, of which a mask leaves as many as the list takes, and more."""
import math

import numpy as np
import pytest
import torch

from test_gpu_sample import check, us

pytestmark = pytest.mark.gpu


def among_others(V, R, left, none, kind, pad, start, seed=0):
    """R rows of V logits, `none` but for `left` of them, from column `start` of a buffer that holds much larger ones everywhere else."""
    g = torch.Generator().manual_seed(seed + V + left)
    x = torch.full((R, V), none)
    for r in range(R):
        at = torch.randperm(V, generator=g)[:left]
        x[r, at] = 2.5 * torch.randn(left, generator=g)
    wide = torch.full((R + 2, V + pad + start), 90.0, dtype=kind, device="cuda")
    view = wide[1:-1, start:start + V]
    view.copy_(x.to(kind))
    return view


# V: of workgroups of 256, 512 and 1024 threads.  left: fewer than a list takes, all of them, and more
@pytest.mark.parametrize("V,left,k", [(1500, 700, 300), (1500, 1500, 900), (8190, 3000, 1000), (8190, 8190, 5000), (50257, 10000, 3000), (50257, 50257, 20000)])
@pytest.mark.parametrize("T", [math.inf, 1e-38, 1e-45])
@pytest.mark.parametrize("kind,pad,start", [(torch.float32, 0, 0), (torch.float32, 3, 1), (torch.bfloat16, 5, 3)])
def test_one_bin_of_all_tokens(V, left, k, T, kind, pad, start):
    for none in (-math.inf, math.nan):
        x = among_others(V, 5, left, none, kind, pad, start)
        check(x, T=T, k=k, u=us(5))
        check(x, T=T, k=k, p=0.7, u=us(5, 1))
        check(x, T=T, k=k, least=0.5, u=us(5, 2))


def test_the_last_row_of_a_buffer():
    """Nothing behind it."""
    for V in (1000, 16388):
        x = torch.empty(V, device="cuda").normal_(generator=torch.Generator(device="cuda").manual_seed(V))[None]
        for T in (math.inf, 1e-38):
            check(x, T=T, k=V - 7, u=us(1))


@pytest.mark.parametrize("V", [3, 40, 3000, 20000])
@pytest.mark.parametrize("T", [1e38, 2e38, math.inf])
def test_tokens_further_below_than_floats_reach(V, T):
    """Several of them, of weights that count."""
    x = torch.full((3, V), -math.inf)
    x[:, [0, V // 2, V - 1]] = torch.tensor([-3.2e38, 3e38, -3e38])
    if V > 3:
        x[1:, 1:4] = torch.tensor([-2.5e38, 1e38, -3.1e38])
        x[2, 4:V // 2] = torch.linspace(-3.3e38, -1e38, V // 2 - 4)
    x = x.cuda()
    for k in (1, 2, 3, 4, 5, 700, 2000):
        check(x, T=T, k=k, u=us(3, k))
        check(x, T=T, k=k, p=0.9, u=us(3, k))
        check(x, T=T, k=k, least=0.1, u=us(3, k))
    check(x, T=T, p=0.95, u=us(3))


@pytest.mark.parametrize("V", [40, 3000, 50257])
@pytest.mark.parametrize("scale,T", [(2.5, 3.3e38), (2.5, math.inf), (1e-20, 1.0), (1e-30, 1e-3), (0.0, 1.0), (1.0, 1e12)])
def test_weights_that_are_all_one(V, scale, T):
    """Where every weight is one in 64 bits, min_p = 1 leaves all tokens, wherever the largest stands."""
    x = (scale * torch.randn((6, V), generator=torch.Generator().manual_seed(V))).cuda()
    # At T = 1e12 weights are below one, by up to 9 / 1e12: many by less than the 2^-38 = 3.6e-12 that the oracle leaves to the weights' last
    # bits, so that every row has a list of tokens there
    unsure = 1.0 if T == 1e12 else 0.02
    check(x, T=T, least=1.0, u=us(6), most_unsure=unsure)
    check(x, T=T, least=1.0, k=V // 2, u=us(6, 1), most_unsure=unsure)
    check(x, T=T, least=1.0, p=0.5, u=us(6, 2), most_unsure=unsure)
    check(x, T=T, least=1.0 - 2.0 ** -24, u=us(6, 3), most_unsure=unsure)
