// Attention of long chunks of new rows over the paged cache: tiles of 128 rows, four waves of 32 rows each.
//
// K and V of 64 tokens at a time go straight into LDS, where all waves read them, while the 64 before are
// worked on.  S^T = K Q^T and O^T = V^T P^T on v_mfma_f32_32x32x16_bf16, as in kv_attention.hip: a lane's column is one row
// of the tile, its two lane halves hold different tokens, and P goes from the first product's result to the second
// one's operand without leaving its lane (16 tokens: 4 h .. 4 h + 3 and 8 + 4 h .. 8 + 4 h + 3 for lane half h).
//
// The running maximum only moves when a score passes it by more than 2^8 in weight, so most steps rescale nothing;
// the weights stay below 2^8 and the sums are the same up to rounding.
#include <limits.h>

#include <algorithm>
#include <cmath>

#include "kv_attention.h"

namespace lora {

namespace {

constexpr int kRows = kLongTile;
constexpr int kTokens = 64;              // of a step
constexpr int kWaves = 4;
constexpr float kSlack = 8.f;            // the maximum's, in powers of two
constexpr float kExact = 4096.f;         // scaled maxima up to which e^(s - m) is formed with one rounding of m

typedef __attribute__((ext_vector_type(16))) float f32x16;

__device__ __align__(16) const unsigned zeros[4] = {0u, 0u, 0u, 0u};

// V^T of 32 columns and 16 tokens.
template <int DP>
__device__ inline bf16x8 v_tile(const uint16_t *s_v, int tokens, int d)
{
    const int l = threadIdx.x & 15, grp = (threadIdx.x & 63) >> 4;
    u32x2 v[2];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const int row = tokens + j * 8 + (grp >> 1) * 4 + (l >> 2);
        v[j] = read_transposed(s_v + row * DP + swizzled<DP>(row, d * 4 + (grp & 1) * 2 + ((l >> 1) & 1)) * 8 + (l & 1) * 4);
    }
    return as_bf16x8(u32x4{v[0][0], v[0][1], v[1][0], v[1][1]});
}

__device__ inline float other_half(float x)
{
    return __shfl_xor(x, 32);
}

template <int DP>
__global__ __launch_bounds__(kWaves * 64, DP > 128 ? 1 : 2) void attend_long_kernel(AttnParams p)
{
    constexpr int KS = DP / 16;          // steps of the first product
    constexpr int DT = DP / 32;          // output tiles of the second
    constexpr int CH = DP / 8;           // 16-byte pieces of a row
    constexpr int RPL = 64 / CH;         // rows that a wave's load covers
    constexpr int NL = kTokens / RPL / kWaves;           // loads of K and of V per wave and step
    constexpr int STAGE = kTokens * DP;  // elements of K or V in LDS
    __shared__ __align__(16) uint16_t s_kv[2][2][STAGE];

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int col = lane & 31, half = lane >> 5;
    const int D = p.c.dim;
    const Plan plan = plan_of<kRows>(p);
    const int n = blockIdx.x;
    if (n >= plan.items) return;
    Seq q;
    const Item it = item_of<kRows>(p, plan, n, q);
    const int tile = (it.cuts > 1 ? it.tile : tiles_of<kRows>(p, q) - 1 - it.tile);      // long ranges first
    const Range rg = range_of<kRows>(p, q, tile, plan.chunk);
    if (it.cut >= rg.splits) return;
    const int lo = rg.lo + it.cut * plan.chunk, hi = min(rg.hi, lo + plan.chunk);

    // this lane's row, and the tokens that it, some row and every row of its wave see
    const int r0 = tile * kRows + wave * 32;
    const int n_rows = q.rows * p.group;
    const int r = r0 + col;
    const int i = r / p.group, g = r - i * p.group;
    const bool real = r < n_rows;
    const int64_t t = p.b.row_start[it.s] + i;
    const int qh = it.head * p.group + g;
    const int see_hi = !real ? 0 : p.causal ? min(hi, q.pos0 + i + 1) : hi;
    const int see_lo = p.window ? max(lo, q.pos0 + i - p.window + 1) : lo;
    const int first_i = r0 / p.group, last_i = min(q.rows - 1, (r0 + 31) / p.group);
    const int any_hi = r0 >= n_rows ? 0 : p.causal ? min(hi, q.pos0 + last_i + 1) : hi;
    const int any_lo = p.window ? max(lo, q.pos0 + first_i - p.window + 1) : lo;
    const int all_hi = p.causal ? min(hi, q.pos0 + first_i + 1) : hi;
    const int all_lo = p.window ? max(lo, q.pos0 + last_i - p.window + 1) : lo;

    bf16x8 qf[KS];
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
        const int d = ks * 16 + half * 8;
        u32x4 x = {0u, 0u, 0u, 0u};
        if (real && d < D) x = ld16<false>(p.q + t * p.ldq + (int64_t)qh * D + d);
        qf[ks] = as_bf16x8(x);
    }
    f32x16 o[DT];
#pragma unroll
    for (int d = 0; d < DT; ++d) o[d] = f32x16{};
    float m = -INFINITY, ms = -INFINITY, l = 0.f;      // maximum, the same in powers of two, this lane's part of the sum

    // this wave's loads: rows (wave * NL + j) * RPL + lane / CH of a step, the piece that belongs at place lane % CH
    const int32_t *table = p.b.table + (int64_t)it.s * p.b.max_pages;
    const int place_mask = (1 << p.c.page_shift) - 1;
    const unsigned lds0 = (unsigned)(uintptr_t)(__attribute__((address_space(3))) uint16_t *)&s_kv[0][0][0];
    const uint16_t *kbase = p.c.k + it.head * p.c.head_stride, *vbase = p.c.v + it.head * p.c.head_stride;
    int page[NL];
    const auto token_of = [&](int j0, int j) { return min(j0 + (wave * NL + j) * RPL + lane / CH, hi - 1); };
    const auto fetch_pages = [&](int j0) {
#pragma unroll
        for (int j = 0; j < NL; ++j) page[j] = table[token_of(j0, j) >> p.c.page_shift];
    };
    const auto fetch = [&](int j0, int stage) {
#pragma unroll
        for (int j = 0; j < NL; ++j) {
            const int row = (wave * NL + j) * RPL + lane / CH;
            const int token = token_of(j0, j);
            const int piece = swizzled<DP>(row, lane % CH);
            const int64_t at = checked_page(page[j], p.c.n_pages, p.b.status) * p.c.page_stride +
                               (int64_t)(token & place_mask) * p.c.token_stride + piece * 8;
            const bool in = piece * 8 < D;
            const unsigned to = lds0 + ((stage * 2) * STAGE + (wave * NL + j) * RPL * DP) * 2;
            load_to_lds<false>(in ? (const void *)(kbase + at) : (const void *)zeros, to);
            load_to_lds<false>(in ? (const void *)(vbase + at) : (const void *)zeros, to + STAGE * 2);
        }
    };
    if (lo < hi) {
        fetch_pages(lo);
        fetch(lo, 0);
        fetch_pages(min(lo + kTokens, hi - 1));
    }
    int stage = 0;
    for (int j0 = lo; j0 < hi; j0 += kTokens, stage ^= 1) {
        wait_loads<0>();
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        if (j0 + kTokens < hi) {
            fetch(j0 + kTokens, stage ^ 1);
            fetch_pages(min(j0 + 2 * kTokens, hi - 1));
        }
        if (j0 >= any_hi || j0 + kTokens <= any_lo) continue;
        const uint16_t *s_k = s_kv[stage][0], *s_v = s_kv[stage][1];
        f32x16 s[2] = {f32x16{}, f32x16{}};
#pragma unroll
        for (int ks = 0; ks < KS; ++ks)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int row = h * 32 + col;
                const u32x4 k = *reinterpret_cast<const u32x4 *>(s_k + row * DP + swizzled<DP>(row, ks * 2 + half) * 8);
                s[h] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(k), qf[ks], s[h], 0, 0, 0);
            }
        const bool edge = j0 < all_lo || j0 + kTokens > all_hi;
        if (edge) {
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const int j = j0 + h * 32 + 8 * (e >> 2) + 4 * half + (e & 3);
                    if (j < see_lo || j >= see_hi) s[h][e] = -INFINITY;
                }
        }
        float top = s[0][0];
#pragma unroll
        for (int e = 1; e < 32; ++e) top = fmaxf(top, s[e >> 4][e & 15]);
        top = fmaxf(top, other_half(top));
        const float tops = top * p.scale_log2;
        if (__any(tops > ms + kSlack)) {
            const float now = fmaxf(m, top), now_s = fmaxf(ms, tops);
            const float f = fabsf(now_s) <= kExact ? __builtin_amdgcn_exp2f(ms - now_s)
                                                  : __builtin_amdgcn_exp2f((m - (now == -INFINITY ? 0.f : now)) * p.scale_log2);
            const float keep = now == -INFINITY ? 1.f : f;
            l *= keep;
#pragma unroll
            for (int d = 0; d < DT; ++d) o[d] *= keep;
            m = now;
            ms = now_s;
        }
        float mul = p.scale_log2, sub = ms == -INFINITY ? 0.f : ms;
        if (__any(fabsf(sub) > kExact)) {         // scores so large that their scaled difference has to be exact
            const float ref = m == -INFINITY ? 0.f : m;
#pragma unroll
            for (int e = 0; e < 32; ++e) s[e >> 4][e & 15] = (s[e >> 4][e & 15] - ref) * p.scale_log2;
            mul = 1.f;
            sub = 0.f;
        }
        bf16x8 pf[4];
        float sum = 0.f;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            u32x4 w;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float a = __builtin_amdgcn_exp2f(fmaf(s[k >> 1][(k & 1) * 8 + 2 * e], mul, -sub));
                const float b = __builtin_amdgcn_exp2f(fmaf(s[k >> 1][(k & 1) * 8 + 2 * e + 1], mul, -sub));
                sum += a + b;
                w[e] = pack_bf16_rne(a, b);
            }
            pf[k] = as_bf16x8(w);
        }
        l += sum;
        // V of a token that some rows must not see may be no number: 0 * NaN would reach them
        bool odd = false;
        if (edge) {
#pragma unroll 1
            for (int k = 0; k < 4; ++k)
#pragma unroll
                for (int d = 0; d < DT; ++d) odd |= not_finite(__builtin_bit_cast(u32x4, v_tile<DP>(s_v, k * 16, d)));
            odd = __any(odd);
        }
        if (!odd) {
#pragma unroll
            for (int k = 0; k < 4; ++k)
#pragma unroll
                for (int d = 0; d < DT; ++d)
                    o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v_tile<DP>(s_v, k * 16, d), pf[k], o[d], 0, 0, 0);
        } else {
#pragma unroll
            for (int k = 0; k < 4; ++k)
#pragma unroll
                for (int d = 0; d < DT; ++d)
                    o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(finite_part(v_tile<DP>(s_v, k * 16, d)), pf[k], o[d], 0, 0, 0);
            // the rest reaches the rows that see it: whatever the weight, infinity or NaN stays what it is
#pragma unroll 1
            for (int j = 0; j < kTokens; ++j) {
                if (j0 + j < see_lo || j0 + j >= see_hi) continue;
#pragma unroll
                for (int d = 0; d < DT; ++d)
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        const int c = d * 32 + 8 * (e >> 2) + 4 * half + (e & 3);
                        o[d][e] += odd_part(s_v[j * DP + swizzled<DP>(j, c >> 3) * 8 + (c & 7)]);
                    }
            }
        }
    }
    l += other_half(l);
    if (!real) return;
    const float ref = ms == -INFINITY ? 0.f : ms;
    if (rg.splits == 1) {
        const float norm = l == 0.f ? 0.f : 1.f / l;
        uint16_t *out = p.out + t * p.ldo + (int64_t)qh * D;
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int c = d * 32 + e * 8 + half * 4;
                if (c >= D) continue;
                u32x2 b;
                b[0] = pack_bf16_rne(o[d][4 * e] * norm, o[d][4 * e + 1] * norm);
                b[1] = pack_bf16_rne(o[d][4 * e + 2] * norm, o[d][4 * e + 3] * norm);
                *reinterpret_cast<u32x2 *>(out + c) = b;
            }
        if (p.lse && half == 0) p.lse[t * p.heads + qh] = l == 0.f ? -INFINITY : (ref + __builtin_amdgcn_logf(l)) * kLn2;
    } else {
        const int64_t at = (int64_t)it.slot * kRows + wave * 32 + col;
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int c = d * 32 + e * 8 + half * 4;
                if (c < D) st16f(p.long_o + at * D + c, f32x4{o[d][4 * e], o[d][4 * e + 1], o[d][4 * e + 2], o[d][4 * e + 3]});
            }
        if (half == 0) {
            p.long_ml[at * 2] = m;
            p.long_ml[at * 2 + 1] = l;
        }
    }
}

}  // namespace

hipError_t launch_attend_long(const AttnParams &p, int max_items, hipStream_t s)
{
    const dim3 grid(max_items), block(kWaves * 64);
    if (p.c.dim <= 64) hipLaunchKernelGGL(attend_long_kernel<64>, grid, block, 0, s, p);
    else if (p.c.dim <= 128) hipLaunchKernelGGL(attend_long_kernel<128>, grid, block, 0, s, p);
    else hipLaunchKernelGGL(attend_long_kernel<256>, grid, block, 0, s, p);
    return hipGetLastError();
}

}  // namespace lora
