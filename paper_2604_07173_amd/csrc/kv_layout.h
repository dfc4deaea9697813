// How a cache's pages lie in memory.  Host only, plain C++.
#pragma once
#include <stdint.h>

#include "../../include/lora_attn.h"

namespace lora {

// A page as outer x inner runs of `run` elements that lie together; strides in elements.
struct PageRuns {
    int run, inner, outer;
    int64_t inner_stride, outer_stride;
};

// Of heads and tokens the one with the smaller stride is inside.  A run is counted in 32 bits: heads and tokens of a page
// that would be longer in one stay apart.
inline PageRuns page_runs(const lora_kv_cache &c)
{
    const bool token_in = c.token_stride <= c.head_stride;
    PageRuns p;
    p.run = c.head_dim;
    p.inner = token_in ? c.page_size : c.n_heads;
    p.outer = token_in ? c.n_heads : c.page_size;
    p.inner_stride = token_in ? c.token_stride : c.head_stride;
    p.outer_stride = token_in ? c.head_stride : c.token_stride;
    if (p.inner_stride == p.run || p.inner == 1) {
        p.run *= p.inner;
        p.inner = p.outer;
        p.inner_stride = p.outer_stride;
        p.outer = 1;
        if (p.inner_stride == p.run && (int64_t)p.run * p.inner <= INT32_MAX) {
            p.run *= p.inner;
            p.inner = 1;
        }
    }
    return p;
}

}  // namespace lora
