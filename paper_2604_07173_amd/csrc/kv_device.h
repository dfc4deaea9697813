// Device-side helpers of the paged cache.
#pragma once
#include "kv_internal.h"
#include "lora_device.h"

namespace lora {

// Last index i of a non-decreasing array a[0 .. n) with a[i] <= x, found by a whole wave: 64 values are
// compared at a time, so up to 64 entries take one load and up to 4096 two.  a[0] <= x is taken for granted.
__device__ inline int wave_find(const int32_t *a, int n, int x)
{
    const int lane = threadIdx.x & 63;
    int lo = 0;
    while (n > 1) {
        const int step = (n + 63) >> 6;
        const int i = lane * step;
        const bool le = i < n && a[lo + min(i, n - 1)] <= x;
        const int k = max(0, (int)__popcll(__ballot(le)) - 1);
        lo += k * step;
        n = min(step, n - k * step);
    }
    return lo;
}

// A value that is the same in every lane, where the compiler cannot know it.
__device__ inline int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }

// Inclusive prefix sum over the wave, in six steps of the lanes' own exchange paths (no trip through LDS).
template <class T>
__device__ inline T wave_scan(T x)
{
    static_assert(sizeof(T) == 4, "one register");
#define LORA_SCAN_STEP(CTRL, ROWS) \
    x += __builtin_bit_cast(T, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), CTRL, ROWS, 0xf, false));
    LORA_SCAN_STEP(0x111, 0xf)            // row_shr 1, 2, 4, 8: within 16 lanes
    LORA_SCAN_STEP(0x112, 0xf)
    LORA_SCAN_STEP(0x114, 0xf)
    LORA_SCAN_STEP(0x118, 0xf)
    LORA_SCAN_STEP(0x142, 0xa)            // the last lane of rows 0 and 2 to rows 1 and 3
    LORA_SCAN_STEP(0x143, 0xc)            // lane 31 to the upper half
#undef LORA_SCAN_STEP
    return x;
}

template <class T>
__device__ inline T last_lane(T x)
{
    return __builtin_bit_cast(T, __builtin_amdgcn_readlane(__builtin_bit_cast(int, x), 63));
}

}  // namespace lora
