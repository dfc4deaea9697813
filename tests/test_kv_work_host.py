"""The grid of long tiles (compiled for the CPU with g++): as many workgroups as any batch of that many rows may need, whatever its
lengths and however wrong `max_rows` is, within what a launch may have."""
import os
import subprocess
import tempfile

import numpy as np
import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SRC = r'''
#include <cstdio>
#include "kv_work.h"
int main()
{
    int a[6];
    while (scanf("%d %d %d %d %d %d", a, a + 1, a + 2, a + 3, a + 4, a + 5) == 6) {
        const lora::Kinds k = lora::kinds_of(a[0], a[1], a[2], a[3], a[4], a[5]);
        printf("%d %d %d %lld\n", k.has_short, k.has_long, k.limit, (long long)k.long_items);
    }
    printf("%d %d %d\n", lora::kLongTile, lora::kLongTarget, lora::kLongMinSplit);
    return 0;
}
'''


@pytest.fixture(scope="module")
def kinds():
    d = tempfile.mkdtemp()
    src, exe = os.path.join(d, "work_probe.cpp"), os.path.join(d, "work_probe")
    open(src, "w").write(SRC)
    subprocess.check_call(["g++", "-O1", "-std=c++17", "-I", os.path.join(ROOT, "paper_2604_07173_amd", "csrc"), src, "-o", exe])

    def call(cases):
        text = "\n".join(" ".join(map(str, c)) for c in cases)
        lines = subprocess.run([exe], input=text, capture_output=True, text=True, check=True).stdout.split("\n")
        out = [tuple(map(int, l.split())) for l in lines if l]
        return out[:-1], out[-1]
    return call


ROWS = 1 << 20          # rows and sequences of a batch, and rows x heads, at most
ROWS_HEADS = 1 << 29


def test_the_launch_stays_within_the_thread_limit(kinds):
    cases = []
    for heads, kv in [(1, 1), (8, 1), (64, 1), (32, 8), (64, 64), (512, 512), (2048, 32), (33, 1), (1024, 1024), (32768, 32768), (32768, 512)]:
        most = min(ROWS, ROWS_HEADS // heads)
        for n_rows in {most, most - 1, most // 2, most // 33 * 33, 1}:
            for n_seqs in {1, n_rows, max(1, n_rows // 2), max(1, n_rows // 33), max(1, n_rows // 65), ROWS}:
                for max_rows in {0, 1, 2, 33, 65, max(1, n_rows // n_seqs), n_rows}:
                    if n_rows:
                        cases.append((n_seqs, n_rows, max_rows, heads, kv, 8))
    got, _ = kinds(cases)
    for c, (has_short, has_long, limit, items) in zip(cases, got):
        assert has_short or has_long
        if has_long:
            assert 0 < items * 256 < 1 << 32, (c, items)                # workgroups of 256 threads


def needed(rows, lens, heads, kv, limit, tile, target, min_split):
    """Work items of long tiles as the plan on the device makes them, without a window."""
    group = heads // kv
    n = rows * group
    tiles = np.where(n > limit, -(-n // tile), 0)
    work = float((tiles * lens).sum()) * kv * 1.25 / target
    chunk = min_split if work < min_split else (int(work) + 128) >> 7 << 7
    cuts = np.where(lens <= chunk, 1, -(-lens // chunk))
    return int((tiles * cuts).sum()) * kv


def test_there_is_a_workgroup_for_every_item(kinds):
    rng = np.random.default_rng(5)
    cases, batches = [], []
    for _ in range(4000):
        kv = int(rng.choice([1, 2, 8, 64]))
        heads = kv * int(rng.choice([1, 2, 4, 5, 33, 64]))
        n_seqs = int(2 ** rng.uniform(0, 9))
        kind = rng.integers(4)
        if kind == 0:
            rows = np.full(n_seqs, rng.integers(1, 200))
        elif kind == 1:                              # as many sequences as can be just above a limit
            rows = np.full(n_seqs, int(rng.choice([33, 65])) // (heads // kv) + 1)
        elif kind == 2:
            rows = rng.integers(0, 200, n_seqs)
        else:
            rows = np.ones(n_seqs, int)
            rows[rng.integers(n_seqs)] = rng.integers(1, 3000)
        rows[rng.integers(n_seqs)] += 1
        lens = (2 ** rng.uniform(0, 15, n_seqs)).astype(np.int64)
        total = int(rows.sum())
        says = int(rng.choice([0, rows.max(), 1, max(1, total // n_seqs), total]))
        cases.append((n_seqs, total, says, heads, kv, 64))
        batches.append((rows.astype(np.int64), lens))
    got, (tile, target, split) = kinds(cases)
    for c, (rows, lens), (_, has_long, limit, items) in zip(cases, batches, got):
        if has_long:
            assert needed(rows, lens, c[3], c[4], limit, tile, target, split) <= items, c


def test_batches_of_few_rows_start_few_workgroups(kinds):
    """Decoding users beside at most a few long chunks, or an unknown longest one: no workgroup for every user."""
    cases = [(256, 256, 0, 32, 8, 128), (64, 64, 0, 32, 8, 128), (1000, 2000, 900, 32, 8, 128)]
    got, (tile, target, _) = kinds(cases)
    for c, (_, has_long, limit, items) in zip(cases, got):
        n = c[1] * c[3] // c[4]
        assert has_long and items <= target + c[4] * (n // (limit + 1) + n // tile), (c, items)
