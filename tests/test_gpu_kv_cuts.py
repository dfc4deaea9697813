"""Attention where the plan comes from memory (more than 256 sequences) and tiles are cut: the parts of short tiles and of long ones,
their places in the workspace, and the join, for widths of either kind."""
import numpy as np
import pytest

from kv_common import KvCase, attend, attention64, check_attention

pytestmark = pytest.mark.gpu


def run(case, **kw):
    case.device()
    check_attention(case, attend(case, case.dim ** -0.5, **kw), attention64(case, case.dim ** -0.5, **kw))


def uneven(n, seed):
    """Lengths and rows of n sequences: most short or empty, a few of up to 3000 tokens with one to nine rows."""
    rng = np.random.default_rng(seed)
    lens = rng.integers(0, 40, n)
    rows = np.minimum(lens, rng.integers(0, 3, n))
    for s in rng.choice(n, 6, replace=False):
        lens[s] = rng.integers(600, 3000)
        rows[s] = rng.integers(1, 10)
    return rows.tolist(), lens.tolist()


@pytest.mark.parametrize("n", [257, 300, 1100, 2100])
@pytest.mark.parametrize("kw", [dict(), dict(window=700), dict(causal=False)])
def test_cut_short_tiles_of_many_sequences(n, kw):
    rows, lens = uneven(n, n)
    run(KvCase(rows, lens, 4, 2, 64, seed=n), **kw)
    run(KvCase(rows, lens, 4, 2, 64, seed=n, max_rows=0), **kw)


@pytest.mark.parametrize("n,dim", [(300, 128), (1100, 64), (2100, 80)])
@pytest.mark.parametrize("kw", [dict(), dict(window=900), dict(causal=False)])
def test_cut_long_tiles_of_many_sequences(n, dim, kw):
    """Chunks of rows at the batch's start, in its middle, and as its last sequences."""
    rows, lens = uneven(n, n + 1)
    for s, m, length in ((0, 130, 1600), (n // 2, 100, 2500), (n - 2, 40, 700), (n - 1, 150, 1800)):
        rows[s], lens[s] = m, length
    run(KvCase(rows, lens, 4, 2, dim, seed=n), **kw)


def test_cut_long_tiles_alone_of_many_sequences():
    """As many rows in every sequence: no short tiles."""
    lens = [45] * 290 + [900] * 3 + [2000] * 2
    run(KvCase([40] * 295, lens, 2, 2, 64, seed=5))


@pytest.mark.parametrize("heads,kv,dim", [(4, 2, 64), (6, 2, 80), (2, 1, 40), (4, 2, 256), (4, 1, 200), (12, 2, 96), (3, 3, 136)])
@pytest.mark.parametrize("kw", [dict(), dict(window=800), dict(causal=False)])
def test_cut_long_tiles_of_every_width(heads, kv, dim, kw):
    run(KvCase([130, 1, 70], [1900, 800, 1300], heads, kv, dim, seed=dim), **kw)
    run(KvCase([150], [1700], heads, kv, dim, slot_major=True, seed=dim + 1), **kw)
