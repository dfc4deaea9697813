// Attention of new rows over the paged cache, for few rows per sequence (decoding, drafted tokens).
//
// A tile is 16 rows of one sequence and one key/value head: row r is query head r % group of new token
// r / group, so the heads that share K and V share their loads.  A work item is a tile and a range of its visible
// tokens; a long range is cut into items that run in parallel and are joined by a second kernel.  Within
// an item four waves take turns at blocks of 32 tokens, each with a running maximum m, sum l and output O:
//   m' = max(m, s),  l' = l e^(m - m') + sum e^(s - m'),  O' = O e^(m - m') + e^(s - m') V,
// and are joined at the end through LDS by the same rule.
//
// S^T = K Q^T and O^T = V^T P^T on v_mfma_f32_16x16x32_bf16: a lane's column is one row of the tile, so the maximum,
// the sum and the rescaling need no exchange but one across the four lane groups, and the lanes that hold
// P as the result of the first product hold it as the operand of the second: the 32 tokens go into
// the second product in the order in which the first left them (group g: tokens 4g .. 4g+3 and
// 16+4g .. 16+4g+3).  V is read transposed from LDS in that order (ds_read_b64_tr_b16).
#include <limits.h>

#include <algorithm>
#include <cmath>

#include "kv_attention.h"

namespace lora {

namespace {

constexpr int kWaves = 4;
constexpr int kBlock = 32;               // tokens of a wave's step
constexpr int kRows = kShortTile;
constexpr int kPlanThreads = 1024;

// The plan of batches of more than kInlineSeqs sequences.
__global__ __launch_bounds__(kPlanThreads) void plan_kernel(AttnParams p) { make_plan<kPlanThreads>(p, p.plan, true); }

// V^T of 16 columns and a block's 32 tokens, in the order of the second product (see above).
template <int DP>
__device__ inline u32x4 v_tile(const uint16_t *s_v, int d)
{
    const int col = threadIdx.x & 15, grp = (threadIdx.x & 63) >> 4;
    u32x2 v[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int row = h * 16 + grp * 4 + (col >> 2);
        v[h] = read_transposed(s_v + row * DP + swizzled<DP>(row, 2 * d + ((col >> 1) & 1)) * 8 + (col & 1) * 4);
    }
    return u32x4{v[0][0], v[0][1], v[1][0], v[1][1]};
}

// DP: width of a head rounded up to what the products take; loads beyond the head's own width give zeros.
template <int DP>
__global__ __launch_bounds__(kWaves * 64) void attend_kernel(AttnParams p)
{
    constexpr int KS = DP / 32;          // steps of the first product
    constexpr int DT = DP / 16;          // output tiles of the second
    constexpr int CH = DP / 8;           // 16-byte pieces of a row of V
    constexpr int RPL = 64 / CH;         // rows of V that a wave's load covers
    constexpr int VL = kBlock / RPL;     // loads of V per step
    constexpr int OS = DP + 4;           // floats of a row of O in LDS
    constexpr int kVBytes = kWaves * kBlock * DP * 2, kOBytes = kWaves * kRows * OS * 4;
    __shared__ __align__(16) char s_mem[kVBytes > kOBytes ? kVBytes : kOBytes];
    __shared__ float s_m[kWaves][kRows], s_l[kWaves][kRows];

    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int col = lane & 15, grp = lane >> 4;
    __shared__ int32_t s_plan[kInlineWords];
    const int32_t *plan = plan_of(p, s_plan);
    const int items = plan[kItemsShort];
    const int D = p.c.dim;
    uint16_t *s_v = reinterpret_cast<uint16_t *>(s_mem) + wave * kBlock * DP;
    float *s_o = reinterpret_cast<float *>(s_mem);

    for (int n = blockIdx.x; n < items; n += gridDim.x) {
        Seq q;
        const Item it = item_of<kRows>(p, plan, n, q);
        const int s = it.s, head = it.head, tile = it.tile, cut = it.cut;
        const Range rg = range_of<kRows>(p, q, tile, plan[kChunkShort]);
        if (cut >= rg.splits) continue;
        const int lo = rg.lo + cut * rg.each, hi = min(rg.hi, lo + rg.each);

        // this lane's row
        const int r = tile * kRows + col;
        const int i = r / p.group, g = r - i * p.group;
        const bool real = r < q.rows * p.group;
        const int64_t t = p.b.row_start[s] + i;
        const int qh = head * p.group + g;
        const int see_hi = !real ? 0 : p.causal ? min(hi, q.pos0 + i + 1) : hi;
        const int see_lo = p.window ? max(lo, q.pos0 + i - p.window + 1) : lo;
        bf16x8 qf[KS];
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            const int d = ks * 32 + grp * 8;
            u32x4 x = {0u, 0u, 0u, 0u};
            if (real && d < D) x = ld16<false>(p.q + t * p.ldq + (int64_t)qh * D + d);
            qf[ks] = as_bf16x8(x);
        }

        // tokens that every row of the tile sees; a block that goes beyond them has to be masked
        const int all_lo = p.window ? q.pos0 + min(q.rows - 1, (tile * kRows + kRows - 1) / p.group) - p.window + 1 : lo;
        const int all_hi = p.causal ? min(hi, q.pos0 + tile * kRows / p.group + 1) : hi;

        f32x4 o[DT];
#pragma unroll
        for (int d = 0; d < DT; ++d) o[d] = f32x4{0.f, 0.f, 0.f, 0.f};
        float m = -INFINITY, l = 0.f;
        const int32_t *table = p.b.table + (int64_t)s * p.b.max_pages;
        const int place_mask = (1 << p.c.page_shift) - 1;
        const uint16_t *kbase = p.c.k + head * p.c.head_stride, *vbase = p.c.v + head * p.c.head_stride;

        for (int j0 = lo + wave * kBlock; j0 < hi; j0 += kWaves * kBlock) {
            // the block's tokens; those past the range are read as its last one and masked below
            const int mine = min(j0 + (lane & 31), hi - 1);
            const int page = checked_page(table[mine >> p.c.page_shift], p.c.n_pages, p.b.status);
            const int64_t at = page * p.c.page_stride + (int64_t)(mine & place_mask) * p.c.token_stride;
            u32x4 kx[2][KS], vx[VL];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int64_t row = __shfl(at, h * 16 + col);
#pragma unroll
                for (int ks = 0; ks < KS; ++ks) {
                    const int d = ks * 32 + grp * 8;
                    kx[h][ks] = d < D ? ld16<false>(kbase + row + d) : u32x4{0u, 0u, 0u, 0u};
                }
            }
#pragma unroll
            for (int n = 0; n < VL; ++n) {
                const int64_t row = __shfl(at, n * RPL + lane / CH);
                const int d = (lane % CH) * 8;
                vx[n] = d < D ? ld16<false>(vbase + row + d) : u32x4{0u, 0u, 0u, 0u};
            }
            __builtin_amdgcn_wave_barrier();
#pragma unroll
            for (int n = 0; n < VL; ++n) {
                const int row = n * RPL + lane / CH;
                *reinterpret_cast<u32x4 *>(s_v + row * DP + swizzled<DP>(row, lane % CH) * 8) = vx[n];
            }
            f32x4 sc[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                sc[h] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int ks = 0; ks < KS; ++ks)
                    sc[h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(kx[h][ks]), qf[ks], sc[h], 0, 0, 0);
            }
            float x[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = sc[e >> 2][e & 3];
            const bool edge = j0 < all_lo || j0 + kBlock > all_hi;
            if (edge) {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int j = j0 + (e >> 2) * 16 + grp * 4 + (e & 3);
                    if (j < see_lo || j >= see_hi) x[e] = -INFINITY;
                }
            }
            float top = x[0];
#pragma unroll
            for (int e = 1; e < 8; ++e) top = fmaxf(top, x[e]);
            top = fmaxf(top, __shfl_xor(top, 16));
            top = fmaxf(top, __shfl_xor(top, 32));
            const float now = fmaxf(m, top);
            // the difference is taken before the scale: exact where it matters, however large the scores are
            const float ref = now == -INFINITY ? 0.f : now;
            const float shrink = __builtin_amdgcn_exp2f((m - ref) * p.scale_log2);
            float w[8], sum = 0.f;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                w[e] = __builtin_amdgcn_exp2f((x[e] - ref) * p.scale_log2);
                sum += w[e];
            }
            l = l * shrink + sum;
            m = now;
            u32x4 pk;
#pragma unroll
            for (int e = 0; e < 4; ++e) pk[e] = pack_bf16_rne(w[2 * e], w[2 * e + 1]);
            const bf16x8 pf = as_bf16x8(pk);
            __builtin_amdgcn_wave_barrier();
            // V of a token that some rows must not see may be no number: 0 * NaN would reach them
            bool odd = false;
            if (edge) {
#pragma unroll
                for (int d = 0; d < DT; ++d) odd |= not_finite(v_tile<DP>(s_v, d));
                odd = __any(odd);
            }
            if (!odd) {
#pragma unroll
                for (int d = 0; d < DT; ++d)
                    o[d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(v_tile<DP>(s_v, d)), pf, o[d] * shrink, 0, 0, 0);
            } else {
#pragma unroll
                for (int d = 0; d < DT; ++d)
                    o[d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(finite_part(as_bf16x8(v_tile<DP>(s_v, d))), pf, o[d] * shrink, 0, 0, 0);
                // the rest reaches the rows that see it: whatever the weight, infinity or NaN stays what it is
#pragma unroll 1
                for (int j = 0; j < kBlock; ++j) {
                    if (j0 + j < see_lo || j0 + j >= see_hi) continue;
#pragma unroll
                    for (int d = 0; d < DT; ++d)
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const int c = d * 16 + grp * 4 + e;
                            o[d][e] += odd_part(s_v[j * DP + swizzled<DP>(j, c >> 3) * 8 + (c & 7)]);
                        }
                }
            }
            __builtin_amdgcn_wave_barrier();
        }
        // the four waves' parts of the range
        l += __shfl_xor(l, 16);
        l += __shfl_xor(l, 32);
        __syncthreads();
#pragma unroll
        for (int d = 0; d < DT; ++d)
            *reinterpret_cast<f32x4 *>(s_o + (wave * kRows + col) * OS + d * 16 + grp * 4) = o[d];
        if (grp == 0) s_m[wave][col] = m, s_l[wave][col] = l;
        __syncthreads();
        const int row = threadIdx.x >> 4;
        const int rr = tile * kRows + row;
        if (rr < q.rows * p.group) {
            float top = s_m[0][row];
#pragma unroll
            for (int w = 1; w < kWaves; ++w) top = fmaxf(top, s_m[w][row]);
            const float ref = top == -INFINITY ? 0.f : top;
            float f[kWaves], total = 0.f;
#pragma unroll
            for (int w = 0; w < kWaves; ++w) {
                f[w] = __builtin_amdgcn_exp2f((s_m[w][row] - ref) * p.scale_log2);
                total += f[w] * s_l[w][row];
            }
            const int ri = rr / p.group;
            const int64_t rt = p.b.row_start[s] + ri;
            const int rh = head * p.group + rr - ri * p.group;
            const bool whole = rg.splits == 1;
            const float norm = !whole ? 1.f : total == 0.f ? 0.f : 1.f / total;
            for (int d = (threadIdx.x & 15) * 4; d < D; d += 64) {
                f32x4 sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int w = 0; w < kWaves; ++w)
                    sum += *reinterpret_cast<f32x4 *>(s_o + (w * kRows + row) * OS + d) * f[w];
                if (whole) {
                    sum *= norm;
                    u32x2 b;
                    b[0] = pack_bf16_rne(sum[0], sum[1]);
                    b[1] = pack_bf16_rne(sum[2], sum[3]);
                    *reinterpret_cast<u32x2 *>(p.out + rt * p.ldo + (int64_t)rh * D + d) = b;
                } else {
                    st16f(p.part_o + ((int64_t)it.slot * kRows + row) * D + d, sum);
                }
            }
            if ((threadIdx.x & 15) == 0) {
                if (!whole) {
                    p.part_ml[((int64_t)it.slot * kRows + row) * 2] = top;
                    p.part_ml[((int64_t)it.slot * kRows + row) * 2 + 1] = total;
                } else if (p.lse) {
                    p.lse[rt * p.heads + rh] = total == 0.f ? -INFINITY : (ref * p.scale_log2 + __builtin_amdgcn_logf(total)) * kLn2;
                }
            }
        }
        __syncthreads();                 // LDS is V's again
    }
}

// Joins the cuts of rows whose range was cut, by the rule of the running softmax: a wave per row and head.  Lanes look at
// 64 cuts' maxima and sums at a time, and hand their factors on to the lanes that add up the outputs: DP / 4 lanes take one
// cut's 16 bytes each, eight cuts are on their way at once.
template <int DP>
__global__ __launch_bounds__(256) void join_kernel(AttnParams p)
{
    constexpr int LANES = DP / 4, SETS = 64 / LANES, DEEP = 8;
    __shared__ int32_t s_plan[kInlineWords];
    const int32_t *plan = plan_of(p, s_plan);
    const int units = plan[kJoinUnits];
    const int lane = threadIdx.x & 63, set = lane / LANES, d = (lane % LANES) * 4;
    for (int u = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + (threadIdx.x >> 6)); u < units; u += gridDim.x * 4) {
        const int32_t *base = plan + kPlanHead + kBaseJoin * p.b.n_seqs;
        const int s = wave_find(base, p.b.n_seqs, u);
        const int left = u - base[s];
        const int i = left / p.heads, qh = left - i * p.heads;
        const Seq q = seq_of(p.b, s);
        const int head = qh / p.group;
        const int r = i * p.group + qh - head * p.group;
        const bool is_short = tiles_of<kShortTile>(p, q) > 0;
        const int R = is_short ? kShortTile : kLongTile, chunk = plan[is_short ? kChunkShort : kChunkLong];
        const int tile = r / R;
        const int cuts = is_short ? range_of<kShortTile>(p, q, tile, chunk).splits : range_of<kLongTile>(p, q, tile, chunk).splits;
        if (cuts == 1) continue;
        const int most = splits_of(is_short ? reach_of<kShortTile>(p, q) : reach_of<kLongTile>(p, q), chunk);
        const int slot = plan[kPlanHead + (is_short ? kSlotShort : kSlotLong) * p.b.n_seqs + s] + tile * most * p.c.n_heads + head;
        const int64_t first = (int64_t)slot * R + r - tile * R, step = (int64_t)p.c.n_heads * R;
        const float *ml = is_short ? p.part_ml : p.long_ml, *po = is_short ? p.part_o : p.long_o;
        const int64_t t = p.b.row_start[s] + i;

        float m = -INFINITY, total = 0.f;
        f32x4 sum = {0.f, 0.f, 0.f, 0.f};
        for (int c0 = 0; c0 < cuts; c0 += 64) {
            const bool have = c0 + lane < cuts;
            const float *at = ml + (first + min(c0 + lane, cuts - 1) * step) * 2;
            const float own_m = have ? at[0] : -INFINITY, own_l = have ? at[1] : 0.f;
            float now = own_m;
#pragma unroll
            for (int x = 32; x; x >>= 1) now = fmaxf(now, __shfl_xor(now, x));
            now = fmaxf(m, now);
            const float ref = now == -INFINITY ? 0.f : now;
            const float keep = __builtin_amdgcn_exp2f((m - ref) * p.scale_log2);
            const float f = __builtin_amdgcn_exp2f((own_m - ref) * p.scale_log2);
            float part = f * own_l;
#pragma unroll
            for (int x = 32; x; x >>= 1) part += __shfl_xor(part, x);
            total = total * keep + part;
            sum *= keep;
            m = now;
            const int n = min(64, cuts - c0);
            for (int c = 0; c < n; c += SETS * DEEP) {
                f32x4 x[DEEP];
#pragma unroll
                for (int k = 0; k < DEEP; ++k) {
                    const int cc = c + k * SETS + set;
                    x[k] = cc < n && d < p.c.dim ? ld16f(po + (first + (c0 + cc) * step) * p.c.dim + d) : f32x4{0.f, 0.f, 0.f, 0.f};
                }
#pragma unroll
                for (int k = 0; k < DEEP; ++k) sum += x[k] * __shfl(f, min(c + k * SETS + set, 63));
            }
        }
#pragma unroll
        for (int x = LANES; x < 64; x <<= 1)
#pragma unroll
            for (int e = 0; e < 4; ++e) sum[e] += __shfl_xor(sum[e], x);
        const float norm = total == 0.f ? 0.f : 1.f / total;
        if (set == 0 && d < p.c.dim) {
            u32x2 b;
            b[0] = pack_bf16_rne(sum[0] * norm, sum[1] * norm);
            b[1] = pack_bf16_rne(sum[2] * norm, sum[3] * norm);
            *reinterpret_cast<u32x2 *>(p.out + t * p.ldo + (int64_t)qh * p.c.dim + d) = b;
        }
        if (lane == 0 && p.lse) {
            const float ref = m == -INFINITY ? 0.f : m;
            p.lse[t * p.heads + qh] = total == 0.f ? -INFINITY : (ref * p.scale_log2 + __builtin_amdgcn_logf(total)) * kLn2;
        }
    }
}

size_t up256(size_t n) { return (n + 255) & ~(size_t)255; }

// Which kernels a batch takes, and upper bounds of their work items, from what the host knows.
struct Kinds {
    bool has_short, has_long;
    int limit;                            // rows x group of a sequence that goes in short tiles
    int64_t short_items, long_items;
};

Kinds kinds_of(int n_seqs, int n_rows, int max_rows, int heads, int kv_heads)
{
    const int64_t group = heads / kv_heads;
    const int64_t most = max_rows > 0 ? std::min(max_rows, n_rows) : n_rows;
    Kinds k;
    k.has_long = most * group > kShortLimit;
    k.has_short = !k.has_long || !(max_rows > 0 && (int64_t)max_rows * n_seqs == n_rows);
    // a sequence with more rows than the host thought still has to go somewhere
    k.limit = !k.has_long ? INT_MAX : !k.has_short ? 0 : kShortLimit;
    const int64_t some = std::min(n_seqs, n_rows);
    k.short_items = kShortTarget + kv_heads * (some + n_rows * group / kShortTile);
    k.long_items = kLongTarget + kv_heads * (some + n_rows * group / kLongTile);
    return k;
}

struct Ws {
    size_t plan, short_ml, short_o, long_ml, long_o, bytes;
};

Ws ws_of(int n_seqs, const Kinds &k, int dim)
{
    Ws w;
    w.plan = 0;
    w.short_ml = up256((kPlanHead + kPlanArrays * (size_t)n_seqs) * 4);
    w.short_o = w.short_ml + up256(k.has_short ? 2 * (size_t)kShortTarget * kShortTile * 8 : 0);
    w.long_ml = w.short_o + up256(k.has_short ? 2 * (size_t)kShortTarget * kShortTile * dim * 4 : 0);
    w.long_o = w.long_ml + up256(k.has_long ? 2 * (size_t)kLongTarget * kLongTile * 8 : 0);
    w.bytes = w.long_o + up256(k.has_long ? 2 * (size_t)kLongTarget * kLongTile * dim * 4 : 0);
    return w;
}

}  // namespace

size_t attention_ws_bytes(int n_seqs, int n_rows, int max_rows, int heads, int kv_heads, int dim)
{
    return ws_of(n_seqs, kinds_of(n_seqs, n_rows, max_rows, heads, kv_heads), dim).bytes;
}

hipError_t launch_attention(AttnParams &p, int max_rows, void *ws, hipStream_t s)
{
    const Kinds k = kinds_of(p.b.n_seqs, p.b.n_rows, max_rows, p.heads, p.c.n_heads);
    const Ws at = ws_of(p.b.n_seqs, k, p.c.dim);
    char *w = static_cast<char *>(ws);
    p.plan = reinterpret_cast<int32_t *>(w + at.plan);
    p.part_ml = reinterpret_cast<float *>(w + at.short_ml);
    p.part_o = reinterpret_cast<float *>(w + at.short_o);
    p.long_ml = reinterpret_cast<float *>(w + at.long_ml);
    p.long_o = reinterpret_cast<float *>(w + at.long_o);
    p.short_limit = k.limit;
    if (p.b.n_seqs > kInlineSeqs) hipLaunchKernelGGL(plan_kernel, dim3(1), dim3(kPlanThreads), 0, s, p);
    if (k.has_long) {
        const hipError_t e = launch_attend_long(p, (int)std::min<int64_t>(k.long_items, INT_MAX), s);
        if (e != hipSuccess) return e;
    }
    if (k.has_short) {
        const dim3 grid((unsigned)std::min<int64_t>(k.short_items, 1024)), block(kWaves * 64);
        if (p.c.dim <= 64) hipLaunchKernelGGL(attend_kernel<64>, grid, block, 0, s, p);
        else if (p.c.dim <= 128) hipLaunchKernelGGL(attend_kernel<128>, grid, block, 0, s, p);
        else hipLaunchKernelGGL(attend_kernel<256>, grid, block, 0, s, p);
    }
    if (std::min<int64_t>(p.b.tokens_max, p.window ? (int64_t)p.window + kLongTile : INT_MAX) > kShortMinSplit) {
        // of short tiles at most kShortTarget can be cut, of long ones kLongTarget
        const int64_t units = std::min<int64_t>((int64_t)p.b.n_rows * p.heads, (k.has_short ? kShortTarget * kShortTile : 0) +
                                                                                  (k.has_long ? kLongTarget * kLongTile : 0));
        const dim3 grid((unsigned)std::min<int64_t>((units + 3) / 4, 1024)), block(256);
        if (p.c.dim <= 64) hipLaunchKernelGGL(join_kernel<64>, grid, block, 0, s, p);
        else if (p.c.dim <= 128) hipLaunchKernelGGL(join_kernel<128>, grid, block, 0, s, p);
        else hipLaunchKernelGGL(join_kernel<256>, grid, block, 0, s, p);
    }
    return hipGetLastError();
}

}  // namespace lora
