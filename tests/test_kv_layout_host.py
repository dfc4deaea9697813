"""The runs that a page is copied in (compiled for the CPU with g++): each element of a page once, in 32-bit counts, for pages of any
size that the calls take."""
import os
import subprocess
import tempfile

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SRC = r'''
#include <cstdio>
#include <cstdlib>
#include "kv_layout.h"
int main(int argc, char** argv)
{
    for (int i = 1; i + 4 < argc; i += 5) {
        lora_kv_cache c = {};
        c.n_heads = atoi(argv[i]), c.page_size = atoi(argv[i + 1]), c.head_dim = atoi(argv[i + 2]);
        c.head_stride = atoll(argv[i + 3]), c.token_stride = atoll(argv[i + 4]);
        const lora::PageRuns r = lora::page_runs(c);
        printf("%d %d %d %lld %lld\n", r.run, r.inner, r.outer, (long long)r.inner_stride, (long long)r.outer_stride);
    }
    return 0;
}
'''


@pytest.fixture(scope="module")
def runs():
    d = tempfile.mkdtemp()
    src, exe = os.path.join(d, "runs_probe.cpp"), os.path.join(d, "runs_probe")
    open(src, "w").write(SRC)
    subprocess.check_call(["g++", "-O1", "-std=c++17", "-I", os.path.join(ROOT, "paper_2604_07173_amd", "csrc"), src, "-o", exe])

    def call(*case):
        return tuple(int(v) for v in subprocess.check_output([exe, *map(str, case)]).split())
    return call


@pytest.mark.parametrize("heads,tokens,dim", [(1, 1, 8), (4, 16, 64), (5, 1, 40), (1, 32, 128), (32768, 1024, 64), (32768, 1024, 256),
                                              (8192, 1024, 256), (16384, 512, 248)])
@pytest.mark.parametrize("order", ["head", "token"])
@pytest.mark.parametrize("hole", [0, 8])
def test_runs_cover_a_page(runs, heads, tokens, dim, order, hole):
    inner = dim + hole
    head, token = (tokens * inner, inner) if order == "head" else (inner, heads * inner)
    run, n_in, n_out, s_in, s_out = runs(heads, tokens, dim, head, token)
    assert 0 < run < 2 ** 31 and n_in > 0 and n_out > 0
    assert run * n_in * n_out == heads * tokens * dim
    assert (run // 8) * n_in * n_out <= 2 ** 30                 # 16-byte pieces are numbered in 32 bits
    # first and last element of the first, of the second and of the last run are where the page has them
    where = lambda e: (e // dim // tokens * head + e // dim % tokens * token if order == "head" else                # noqa: E731
                       e // dim // heads * token + e // dim % heads * head) + e % dim
    for r in {0, min(1, n_in * n_out - 1), n_in * n_out - 1}:
        at = r // n_in * s_out + r % n_in * s_in
        assert at == where(r * run) and at + run - 1 == where(r * run + run - 1)
