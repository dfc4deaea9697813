"""Which tokens of a row the sampling kernel lists (compiled for the CPU with g++): those of one bin, and never a place in front of the
row or behind it, whose logits would then be read from memory that is not the row's."""
import math
import os
import subprocess
import tempfile

import numpy as np
import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SRC = r'''
#include <cstdio>
#include <cstdlib>
#include <vector>
#define LORA_HD inline
#include "sample_bins.h"

// The pieces of a workgroup's waves, as the kernel hands them out: 64 lanes' for every step, AHEAD steps at a time, of which those from the
// wave's last step on are no pieces of the row.
template <int VEC, class F>
void each(int threads, int skew, const std::vector<float> &l, F f)
{
    const lora::Pieces<VEC> row{skew, (int)l.size()};
    const int pieces = row.pieces(), steps = (pieces + threads - 1) / threads, ahead = 4;
    for (int w = 0; w < threads / 64; ++w)
        for (int k = 0; k < (steps + ahead - 1) / ahead * ahead; ++k)
            for (int lane = 0; lane < 64; ++lane) {
                const int i = w * steps * 64 + lane + k * 64, load = k < steps ? i : pieces;
                for (int e = 0; e < VEC; ++e) {
                    const int from = row.number(load, e);
                    f(from >= 0 && from < row.vocab ? l[from] : -INFINITY, row.number(i, e));
                }
            }
}

template <int VEC>
void run(int threads, int skew, float T, unsigned want, const std::vector<float> &l)
{
    float top = -INFINITY;
    for (float x : l) top = fmaxf(top, x);
    const int most = 4 * threads;
    const lora::Bins bins = lora::bins_over(48.f, most, T);
    std::vector<unsigned> count(most);
    each<VEC>(threads, skew, l, [&](float x, int) {
        const int b = lora::bin_of(top, x, bins);
        if (b < most) ++count[b];
    });
    int bin = 0;
    for (unsigned sum = 0; bin < most && (sum += count[bin]) < want; ++bin) {}
    printf("%d", bin);
    const lora::Bin it = lora::only_bin(bins, bin);
    each<VEC>(threads, skew, l, [&](float x, int number) {
        if (lora::is_in(top, x, -INFINITY, it)) printf(" %d", number);
    });
    printf("\n");
}

int main(int, char **a)
{
    std::vector<float> l(atoi(a[1]));
    if (fread(l.data(), 4, l.size(), stdin) != l.size()) return 1;
    const int vec = atoi(a[2]), threads = atoi(a[3]), skew = atoi(a[4]);
    if (vec == 4) run<4>(threads, skew, strtof(a[5], nullptr), atoi(a[6]), l);
    else run<8>(threads, skew, strtof(a[5], nullptr), atoi(a[6]), l);
    return 0;
}
'''


@pytest.fixture(scope="module")
def listed():
    d = tempfile.mkdtemp()
    src, exe = os.path.join(d, "bins_probe.cpp"), os.path.join(d, "bins_probe")
    open(src, "w").write(SRC)
    subprocess.check_call(["g++", "-O1", "-std=c++17", "-ffp-contract=off", "-I", os.path.join(ROOT, "paper_2604_07173_amd", "csrc"), src, "-o", exe])

    def call(l, vec, threads, skew, T, k):
        args = [exe, len(l), vec, threads, skew, repr(T), k]
        out = subprocess.run(list(map(str, args)), input=l.astype(np.float32).tobytes(), capture_output=True, check=True).stdout.split()
        return int(out[0]), [int(t) for t in out[1:]]
    return call


def rows(V, left, seed):
    """Logits of which a mask has left some: -inf, or no number, in place of the others."""
    rng = np.random.default_rng(seed)
    l = (2.5 * rng.standard_normal(V)).astype(np.float32)
    for none in (-math.inf, math.nan):
        x = np.full(V, none, np.float32)
        at = rng.permutation(V)[:left]
        x[at] = l[at]
        yield x


@pytest.mark.parametrize("V,threads,vec", [(1000, 256, 4), (1000, 256, 8), (1001, 256, 4), (8190, 512, 8), (8190, 512, 4), (16388, 1024, 4), (20011, 1024, 8), (5, 256, 4)])
@pytest.mark.parametrize("T", [math.inf, 1e-45, 1e-38, 3.6e-37, 1e-3, 1.0, 3e38])
def test_only_tokens_of_the_row_are_listed(listed, V, threads, vec, T):
    for seed, left in enumerate((V, max(1, V // 3), 1)):
        for x in rows(V, left, seed):
            real = np.nonzero(x > -np.inf)[0]                # false for what is no number
            for skew in (0, 1, vec - 1):
                bin, numbers = listed(x, vec, threads, skew, T, max(1, left // 2))
                assert len(set(numbers)) == len(numbers) and np.isin(numbers, real).all(), (skew, left, numbers[:5], numbers[-5:])
                # as many as are wanted are there: in one bin, or where the temperature makes bins useless in the last one
                if T in (math.inf, 1e-45, 1e-38):
                    assert len(numbers) == len(real) and bin == (0 if T == math.inf else 4 * threads)
                assert numbers


@pytest.mark.parametrize("T", [math.inf, 3e38, 2e38, 1e37, 1.0])
def test_no_token_with_a_weight_is_behind_the_bins(listed, T):
    """Also where the difference of two logits is infinite in 32 bits: the bin of the k-th token is found, and no token that stands after all
    of its values is in it."""
    rng = np.random.default_rng(3)
    few = np.array([3e38, -3e38, -3.2e38, -1e38, 3.3e38, -3.4e38, 0.0], np.float32)
    for l in (few[:3], few, (3.4e38 * rng.uniform(-1, 1, 500)).astype(np.float32)):
        order = np.argsort(-l.astype(np.float64), kind="stable")
        weight = np.exp((l.astype(np.float64) - np.float64(l.max())) / np.float64(np.float32(T)))
        for k in range(1, len(l) + 1):
            bin, numbers = listed(l, 4, 256, 1, T, k)
            if weight[order[k - 1]] >= 2.0 ** -47:           # of less it is less than half of what weights are multiples of
                assert bin < 1024 and order[k - 1] in numbers, (k, bin, numbers)
