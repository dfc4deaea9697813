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
#include <algorithm>
#include <cmath>

#include "kv_device.h"

namespace lora {

namespace {

constexpr int kWaves = 4;
constexpr int kBlock = 32;               // tokens of a wave's step
constexpr int kRows = 16;                // rows of a tile
constexpr int kMinSplit = 256;           // tokens of a work item at least, where a range is cut
constexpr int kTargetItems = 2048;       // work items that fill the chip
constexpr int kPlanThreads = 1024;
constexpr float kLn2 = 0.6931471805599453f;

// Device plan: plan[0] = tokens of a work item's range, plan[1 + s] = work items before sequence s.
struct Seq {
    int rows, len, pos0;                 // new rows, length, position of the first new row
};

__device__ inline Seq seq_of(const KvRows &b, int s)
{
    Seq q;
    const int first = min(max(0, b.row_start[s]), b.n_rows);
    q.rows = max(0, min(b.row_start[s + 1], b.n_rows) - first);
    q.len = min(max(0, b.seq_len[s]), b.tokens_max);
    q.pos0 = q.len - q.rows;
    return q;
}

__device__ inline int tiles_of(const Seq &q, int group) { return (q.rows * group + kRows - 1) / kRows; }

// Most tokens that a tile of the sequence sees.
__device__ inline int reach_of(const AttnParams &p, const Seq &q)
{
    if (!p.window) return q.len;
    const int64_t most = (int64_t)p.window - 1 + min(q.rows, kRows / p.group + 2);
    return (int)min((int64_t)q.len, most);
}

__device__ inline int splits_of(int reach, int chunk) { return max(1, (reach + chunk - 1) / chunk); }

// Cuts the ranges so that all work items take about as long, at most max_items of them.
__global__ __launch_bounds__(kPlanThreads) void plan_kernel(AttnParams p)
{
    __shared__ int64_t s_sum[kPlanThreads / 64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int64_t work = 0;
    unsigned bad = 0;
    for (int s = threadIdx.x; s < p.b.n_seqs; s += kPlanThreads) {
        const Seq q = seq_of(p.b, s);
        if (p.b.seq_len[s] != q.len) bad = 1;
        work += (int64_t)tiles_of(q, p.group) * reach_of(p, q);
    }
    if (bad) atomicOr(p.b.status, LORA_STATUS_BAD_LENGTH);
#pragma unroll
    for (int d = 32; d; d >>= 1) work += __shfl_xor(work, d);
    if (lane == 0) s_sum[wave] = work;
    __syncthreads();
    work = 0;
    for (int w = 0; w < kPlanThreads / 64; ++w) work += s_sum[w];
    const int64_t each = (work * p.c.n_heads + kTargetItems - 1) / kTargetItems;
    const int chunk = (int)min(((max(each, (int64_t)kMinSplit) + 127) >> 7) << 7, (int64_t)1 << 30);
    int base = 0;
    for (int s0 = 0; s0 < p.b.n_seqs; s0 += kPlanThreads) {
        const int s = s0 + threadIdx.x;
        int items = 0;
        if (s < p.b.n_seqs) {
            const Seq q = seq_of(p.b, s);
            items = tiles_of(q, p.group) * splits_of(reach_of(p, q), chunk) * p.c.n_heads;
        }
        int v = items;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int o = __shfl_up(v, d);
            if (lane >= d) v += o;
        }
        __syncthreads();
        if (lane == 63) s_sum[wave] = v;
        __syncthreads();
        int total = 0;
        for (int w = 0; w < kPlanThreads / 64; ++w) {
            if (w < wave) v += (int)s_sum[w];
            total += (int)s_sum[w];
        }
        if (s < p.b.n_seqs) p.plan[1 + s] = base + v - items;
        base += total;
    }
    if (threadIdx.x == 0) {
        p.plan[0] = chunk;
        p.plan[1 + p.b.n_seqs] = base;
    }
}

// A tile's tokens: [lo, hi), and of them the part of one of its splits.
struct Range {
    int lo, hi, splits;
};

__device__ inline Range range_of(const AttnParams &p, const Seq &q, int tile, int chunk)
{
    const int i0 = tile * kRows / p.group, i1 = min(q.rows - 1, (tile * kRows + kRows - 1) / p.group);
    Range r;
    r.hi = p.causal ? max(0, min(q.len, q.pos0 + i1 + 1)) : q.len;
    r.lo = p.window ? max(0, q.pos0 + i0 - p.window + 1) : 0;
    if (r.lo >= r.hi) r.lo = r.hi = 0;
    r.splits = splits_of(r.hi - r.lo, chunk);
    return r;
}

// V^T of 16 columns and a block's 32 tokens, in the order of the second product (see above).  A wave's block of V
// lies in LDS as rows of DP; the 16-byte pieces of a row change places by its number, so that the rows that
// are read together lie in different banks.
template <int DP>
__device__ inline int v_piece(int row, int piece) { return piece ^ (2 * (row & 7) & (DP / 8 - 1)); }

template <int DP>
__device__ inline u32x4 v_tile(const uint16_t *s_v, int d)
{
    typedef __attribute__((ext_vector_type(4))) short s16x4;
    typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
    const int col = threadIdx.x & 15, grp = (threadIdx.x & 63) >> 4;
    u32x2 v[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int row = h * 16 + grp * 4 + (col >> 2);
        const uint16_t *at = s_v + row * DP + v_piece<DP>(row, 2 * d + ((col >> 1) & 1)) * 8 + (col & 1) * 4;
        v[h] = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)at));
    }
    return u32x4{v[0][0], v[0][1], v[1][0], v[1][1]};
}

__device__ inline bool not_finite(u32x4 v)       // any of eight bf16
{
    bool r = false;
#pragma unroll
    for (int i = 0; i < 4; ++i) r |= (v[i] & 0x7F800000u) == 0x7F800000u || (v[i] & 0x7F80u) == 0x7F80u;
    return r;
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
    const int chunk = p.plan[0], items = min(p.plan[1 + p.b.n_seqs], p.max_items);
    const int D = p.c.dim;
    uint16_t *s_v = reinterpret_cast<uint16_t *>(s_mem) + wave * kBlock * DP;
    float *s_o = reinterpret_cast<float *>(s_mem);

    for (int item = blockIdx.x; item < items; item += gridDim.x) {
        const int s = wave_find(p.plan + 1, p.b.n_seqs, item);
        const Seq q = seq_of(p.b, s);
        int left = item - p.plan[1 + s];
        const int head = left % p.c.n_heads;
        left /= p.c.n_heads;
        const int cuts = splits_of(reach_of(p, q), chunk);
        const int tile = left / cuts, cut = left - tile * cuts;
        const Range rg = range_of(p, q, tile, chunk);
        if (cut >= rg.splits) continue;
        const int lo = rg.lo + cut * chunk, hi = min(rg.hi, lo + chunk);

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
                *reinterpret_cast<u32x4 *>(s_v + row * DP + v_piece<DP>(row, lane % CH) * 8) = vx[n];
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
                for (int d = 0; d < DT; ++d) o[d] *= shrink;
#pragma unroll 1
                for (int row = 0; row < kRows; ++row) {       // one row at a time, with zeros for what it does not see
                    const int row_lo = __shfl(see_lo, row), row_hi = __shfl(see_hi, row);
#pragma unroll
                    for (int d = 0; d < DT; ++d) {
                        bf16x8 v8 = as_bf16x8(v_tile<DP>(s_v, d));
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            const int j = j0 + (e >> 2) * 16 + grp * 4 + (e & 3);
                            if (j < row_lo || j >= row_hi) v8[e] = (__bf16)0.f;
                        }
                        const f32x4 with = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v8, pf, o[d], 0, 0, 0);
                        if (col == row) o[d] = with;
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
                    st16f(p.part_o + ((int64_t)item * kRows + row) * D + d, sum);
                }
            }
            if ((threadIdx.x & 15) == 0) {
                if (!whole) {
                    p.part_ml[((int64_t)item * kRows + row) * 2] = top;
                    p.part_ml[((int64_t)item * kRows + row) * 2 + 1] = total;
                } else if (p.lse) {
                    p.lse[rt * p.heads + rh] = total == 0.f ? -INFINITY : (ref * p.scale_log2 + __builtin_amdgcn_logf(total)) * kLn2;
                }
            }
        }
        __syncthreads();                 // LDS is V's again
    }
}

// Joins the cuts of rows whose range was cut: a wave per row and head, by the rule of the running softmax.
__global__ __launch_bounds__(256) void join_kernel(AttnParams p)
{
    const int lane = threadIdx.x & 63;
    const int n = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + (threadIdx.x >> 6));
    if (n >= p.b.n_rows * p.heads) return;
    const int t = n / p.heads, qh = n - t * p.heads;
    const int chunk = p.plan[0];
    const int s = wave_find(p.b.row_start, p.b.n_seqs, t);
    const Seq q = seq_of(p.b, s);
    const int head = qh / p.group;
    const int r = (t - p.b.row_start[s]) * p.group + qh - head * p.group;
    const int tile = r / kRows, row = r - tile * kRows;
    const Range rg = range_of(p, q, tile, chunk);
    if (rg.splits == 1) return;
    const int cuts = splits_of(reach_of(p, q), chunk);
    const int64_t first = p.plan[1 + s] + ((int64_t)tile * cuts) * p.c.n_heads + head;
    float m = -INFINITY;
    for (int c = 0; c < rg.splits; ++c) m = fmaxf(m, p.part_ml[((first + c * p.c.n_heads) * kRows + row) * 2]);
    const float ref = m == -INFINITY ? 0.f : m;
    f32x4 sum = {0.f, 0.f, 0.f, 0.f};
    float total = 0.f;
    const int d = lane * 4;
    for (int c = 0; c < rg.splits; ++c) {
        const int64_t at = (first + c * p.c.n_heads) * kRows + row;
        const float f = __builtin_amdgcn_exp2f((p.part_ml[at * 2] - ref) * p.scale_log2);
        total += f * p.part_ml[at * 2 + 1];
        if (d < p.c.dim) sum += ld16f(p.part_o + at * p.c.dim + d) * f;
    }
    const float norm = total == 0.f ? 0.f : 1.f / total;
    if (d < p.c.dim) {
        u32x2 b;
        b[0] = pack_bf16_rne(sum[0] * norm, sum[1] * norm);
        b[1] = pack_bf16_rne(sum[2] * norm, sum[3] * norm);
        *reinterpret_cast<u32x2 *>(p.out + t * p.ldo + (int64_t)qh * p.c.dim + d) = b;
    }
    if (lane == 0 && p.lse) p.lse[(int64_t)t * p.heads + qh] = total == 0.f ? -INFINITY : (ref * p.scale_log2 + __builtin_amdgcn_logf(total)) * kLn2;
}

size_t up256(size_t n) { return (n + 255) & ~(size_t)255; }

// Upper bounds from what the host knows.
int64_t max_items_of(int n_seqs, int n_rows, int heads, int kv_heads)
{
    const int64_t group = heads / kv_heads;
    const int64_t tiles = std::min<int64_t>(n_seqs, n_rows) + (int64_t)n_rows * group / kRows;
    return kTargetItems + tiles * kv_heads;
}

}  // namespace

size_t attention_ws_bytes(int n_seqs, int n_rows, int max_rows, int heads, int kv_heads, int dim)
{
    (void)max_rows;
    const int64_t items = max_items_of(n_seqs, n_rows, heads, kv_heads);
    return up256((size_t)(n_seqs + 2) * 4) + up256((size_t)items * kRows * 8) + (size_t)items * kRows * dim * 4;
}

hipError_t launch_attention(AttnParams &p, int max_rows, void *ws, hipStream_t s)
{
    (void)max_rows;
    p.max_items = (int)max_items_of(p.b.n_seqs, p.b.n_rows, p.heads, p.c.n_heads);
    char *w = static_cast<char *>(ws);
    p.plan = reinterpret_cast<int32_t *>(w);
    w += up256((size_t)(p.b.n_seqs + 2) * 4);
    p.part_ml = reinterpret_cast<float *>(w);
    w += up256((size_t)p.max_items * kRows * 8);
    p.part_o = reinterpret_cast<float *>(w);
    hipLaunchKernelGGL(plan_kernel, dim3(1), dim3(kPlanThreads), 0, s, p);
    const dim3 grid(std::min(p.max_items, 1024)), block(kWaves * 64);
    if (p.c.dim <= 64) hipLaunchKernelGGL(attend_kernel<64>, grid, block, 0, s, p);
    else if (p.c.dim <= 128) hipLaunchKernelGGL(attend_kernel<128>, grid, block, 0, s, p);
    else hipLaunchKernelGGL(attend_kernel<256>, grid, block, 0, s, p);
    const int64_t waves = (int64_t)p.b.n_rows * p.heads;
    hipLaunchKernelGGL(join_kernel, dim3((unsigned)((waves + 3) / 4)), dim3(256), 0, s, p);
    return hipGetLastError();
}

}  // namespace lora
