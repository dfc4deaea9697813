"""The choice of a token by its definition, in 64 bits on the CPU (not a test module)."""
from __future__ import annotations

import math

import numpy as np


def one_row(l, T=1.0, k=0, p=1.0, least=0.0, u=0.5):
    """(token, probability, others): others is None where no border is so near that the weights' last bits decide; else a list of all
    tokens that they may lead to."""
    l = np.asarray(l, np.float64)
    V = len(l)
    l = np.where(np.isnan(l), -math.inf, l)
    top = l.max()
    if top == -math.inf:
        return -1, 0.0, None
    order = np.argsort(-l, kind="stable")
    if not T > 0:
        return int(order[0]), 1.0, None
    if top == math.inf:
        w = (l == top).astype(np.float64)
    else:
        with np.errstate(over="ignore", invalid="ignore"):
            w = np.where(l == -math.inf, 0.0, np.exp((l - top) / T))
    # Each weight is off by half a step of 2^-46 (2^-(62 - bits) for large vocabularies) and by 2^-40 of itself
    step = 2.0 ** -min(46, 62 - max(0, (V - 1).bit_length()))
    w[w < step / 2] = 0.0                            # rounds to zero: never chosen
    sure, moved = True, 0.0                          # moved: weight that may be kept or not
    sorted_w = w[order]
    n = V if k <= 0 else min(V, k)
    off = lambda total: V * step + total * 2.0 ** -38                                       # noqa: E731
    if p < 1:                                        # NaN: no limit
        upto = np.cumsum(sorted_w[:n])
        goal = p * upto[-1]
        near = np.abs(upto - goal).min()
        exact = sorted_w.max() == sorted_w[:n][sorted_w[:n] > 0].min()       # whole multiples of one weight
        if near <= off(upto[-1]) and not (exact and near == 0.0):
            sure = False
            around = np.nonzero(np.abs(upto - goal) <= off(upto[-1]))[0]
            moved += sorted_w[around[0]:around[-1] + 2].sum()
        n = min(n, 1 + int(np.searchsorted(upto, goal, side="left")))
    if least > 0:
        least = min(least, 1.0)
        around = sorted_w[:n]
        sure = sure and not ((np.abs(around - least) < 2.0 ** -38 * least) & (around != least)).any()
        n = min(n, int((sorted_w >= least).sum()))
    kept = np.zeros(V)
    kept[order[:n]] = sorted_w[:n]
    upto = np.cumsum(kept)
    u = 0.0 if not u > 0 else min(u, 1.0 - 2.0 ** -24)
    goal = u * upto[-1]
    token = int(np.argmax(upto > goal))
    edges = upto[kept > 0]
    near = np.abs(edges - goal).min()
    same = kept[kept > 0]
    sure = sure and (near > off(upto[-1]) or same.max() == same.min() == 1.0)
    others = None
    if not sure:                                     # a changed sum of what is kept moves both the goal and the tokens' places
        slack = 2.0 * (off(upto[-1]) + moved)
        others = np.nonzero((upto >= goal - slack) & (upto - kept <= goal + slack) & (w > 0))[0].tolist()
    return token, float(kept[token] / upto[-1]), others
