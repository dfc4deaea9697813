// Attention of new rows over the paged cache, for few rows per sequence (decoding, drafted tokens).
//
// A workgroup's four waves take turns at blocks of 32 tokens of a tile, each with a running maximum m, sum l and output O:
//   m' = max(m, s),  l' = l e^(m - m') + sum e^(s - m'),  O' = O e^(m - m') + e^(s - m') V,
// and are joined at the end through LDS by the same rule, as join_kernel joins the parts of a tile.
//
// S^T = K Q^T and O^T = V^T P^T on v_mfma_f32_16x16x32_bf16: a lane's column is one row of the tile, so the maximum,
// the sum and the rescaling need no exchange but one across the four lane groups, and the lanes that hold
// P as the result of the first product hold it as the operand of the second: the 32 tokens go into
// the second product in the order in which the first left them (group g: tokens 4g .. 4g+3 and
// 16+4g .. 16+4g+3).  The weights, at most 1, are rounded to bf16 there, the type that the products take: an error of 2^-8 of each at
// most, as much as K and V themselves come with; their sum takes them unrounded.  V is read transposed from LDS in that order (ds_read_b64_tr_b16), where it has come straight from
// memory; K goes from memory into the operand registers.
//
// Bound by the reading of K and V from about 100 MB on: 32 / 8 heads of 128, 256 users with 100 to 4000 tokens (1.17 GB) 208 us in
// the kernel and 213 with the join, 5.5 TB/s; three users with 247000 tokens together (1.01 GB) 160 and 169 us, 6.0 TB/s.
// A tile or a fixed cut of one per item, with all loads through registers, took 260 us for either.  Small calls are chains of latencies (one user, 1500 tokens: 7.5 us, 3.5 more for the join).
#include <limits.h>

#include <algorithm>

#include "kv_attention.h"

namespace lora {

namespace {

constexpr int kWaves = 4;
constexpr int kBlock = 32;               // tokens of a wave's step
constexpr int kPlanThreads = 1024;

__device__ __align__(16) const unsigned zeros[4] = {0u, 0u, 0u, 0u};

// The plan of batches of more than kMostInline sequences: as make_plan, by a whole workgroup in rounds.
template <bool S>
__global__ __launch_bounds__(kPlanThreads) void plan_kernel(AttnParams p)
{
    constexpr int WAVES = kPlanThreads / 64;
    __shared__ float s_work[WAVES], s_units[WAVES], s_tiles[WAVES];
    __shared__ int s_sum[kPlanSums][WAVES];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, n = plan_seqs<S>(p);
    float work = 0.f, units = 0.f, tiles = 0.f;
    unsigned bad = 0;
    int group_limit = p.group_limit;
    bool untrue = false;
    if constexpr (S) {
        float all = 0.f, rows = 0.f;
        for (int s = tid; s < p.g.most; s += kPlanThreads) {
            const Seq<S> q = seq_of<S>(p, s);
            all += group_work(p, q);
            rows += (float)q.rows;
        }
        all = wave_scan(all);
        rows = wave_scan(rows);
        if (lane == 63) s_work[wave] = all, s_units[wave] = rows;
        __syncthreads();
        all = rows = 0.f;
        for (int w = 0; w < WAVES; ++w) all += s_work[w], rows += s_units[w];
        __syncthreads();                  // they are used again
        if (all <= kGroupsShort) group_limit = INT_MAX;
        untrue = rows_untrue(p, rows);
    }
    const auto seq = [&](int s) {
        Seq<S> q = seq_of<S>(p, s);
        if (S && q.group && untrue) q.rows = 0;
        return q;
    };
    for (int s = tid; s < n; s += kPlanThreads) {
        const Seq<S> q = seq(s);
        bad |= plan_faults_of<S>(p, s);
        work += (float)tiles_of<kLong>(p, q, group_limit) * (float)reach_of<kLong>(p, q);
        if (S) tiles += (float)tiles_of<kLong>(p, q, group_limit);
        units += (float)(tiles_of<kShort>(p, q, group_limit) * p.c.n_heads) * (float)units_of(reach_of<kShort>(p, q), kUnitShift);
    }
    if (bad) atomicOr(p.b.status, LORA_STATUS_BAD_LENGTH);
    work = wave_scan(work);
    units = wave_scan(units);
    if (S) tiles = wave_scan(tiles);
    if (lane == 63) s_work[wave] = work, s_units[wave] = units, s_tiles[wave] = tiles;
    const bool no_rows = __syncthreads_or(bad & 2);
    work = units = tiles = 0.f;
    for (int w = 0; w < WAVES; ++w) work += s_work[w], units += s_units[w], tiles += s_tiles[w];
    const int shift = unit_shift_of(units);
    const int chunk = p.long_o ? chunk_of<S>(p, work, tiles) : 1 << 30;
    int base[kPlanSums] = {};
    for (int s0 = 0; s0 < n; s0 += kPlanThreads) {
        const int s = s0 + tid;
        int own[kPlanSums] = {}, upto[kPlanSums];
        if (s < n) {
            const Seq<S> q = seq(s);
            if (!no_rows) plan_entry(p, q, shift, chunk, group_limit, own);
            store_seq<S>(p.plan, n, s, q);
        }
        __syncthreads();                  // the round before has been read
#pragma unroll
        for (int a = 0; a < kPlanSums; ++a) {
            upto[a] = wave_scan(own[a]);
            if (lane == 63) s_sum[a][wave] = upto[a];
        }
        __syncthreads();
#pragma unroll
        for (int a = 0; a < kPlanSums; ++a) {
            int total = 0;
            for (int w = 0; w < WAVES; ++w) {
                if (w < wave) upto[a] += s_sum[a][w];
                total += s_sum[a][w];
            }
            if (s < n) p.plan[kPlanHead + (int64_t)a * n + s] = base[a] + upto[a] - own[a];
            base[a] += total;
        }
    }
    if (tid == 0) plan_head(p, p.plan, shift, chunk, base);
    if (S && tid == 0) p.plan[kGroupRows] = group_rows(p, no_rows), p.plan[kGroupLimit] = group_limit;
}

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

// DP: width of a head rounded up to what the products take; FULL: it is the width itself, otherwise zeros stand beyond it.
// MT: 16-row parts of a tile.  BLOCKS: workgroups of a CU.  S: sequences share tokens.
template <int DP, int MT, bool FULL, int BLOCKS, bool S>
__global__ __launch_bounds__(kWaves * 64, BLOCKS) void attend_kernel(AttnParams p)
{
    constexpr int R = 16 * MT;
    constexpr int KS = DP / 32;          // steps of the first product
    constexpr int DT = DP / 16;          // output tiles of the second
    constexpr int CH = DP / 8;           // 16-byte pieces of a row of V
    constexpr int RPL = 64 / CH;         // rows of V that a wave's load covers
    constexpr int VL = kBlock / RPL;     // loads of V per step
    constexpr int OS = DP + 4;           // floats of a row of O in LDS
    constexpr int kVBytes = kWaves * kBlock * DP * 2, kOBytes = kWaves * 16 * OS * 4;
    __shared__ __align__(16) char s_mem[kVBytes > kOBytes ? kVBytes : kOBytes];
    __shared__ float s_m[kWaves][16], s_l[kWaves][16];
    __shared__ int32_t s_plan[kInlineWords<S>];

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int col = lane & 15, grp = lane >> 4;
    const int32_t *plan = plan_of<S>(p, s_plan);
    const int D = FULL ? DP : p.c.dim;
    uint16_t *s_v = reinterpret_cast<uint16_t *>(s_mem) + wave * kBlock * DP;
    const unsigned v_lds = (unsigned)(uintptr_t)(__attribute__((address_space(3))) uint16_t *)s_v;
    float *s_o = reinterpret_cast<float *>(s_mem);

    const int unit_shift = uniform(plan[kUnitTokens]), share = uniform(plan[kShare]);
    const int first = blockIdx.x * share, end = min(first + share, uniform(plan[kUnits]));
    if (first >= end) return;
    const int place_mask = (1 << p.c.page_shift) - 1;

    // A tile of the stretch, or the part of one: its rows, and its tokens [lo, hi).  Q's rows and the first page number are
    // on their way before the tile before is written.
    struct Part {
        Seq<S> q;
        int s, head, tile, lo, hi, units;
        bool whole, later;                // later: not the stretch's first tile
    } part;
    int parts = 0;                        // S: of the tile, if this part begins it, else 0
    int see_lo[MT], see_hi[MT], all_lo, all_hi, page = 0;
    bf16x8 qf[MT][KS];
    const auto take = [&](int u) {
        Seq<S> q;
        const Place pl = place_of<S>(p, plan, u, q);
        const int k0 = u - pl.start, k1 = min(pl.units, k0 + end - u), tile = pl.tile, head = pl.head;
        const Range rg = range_of<kShort>(p, q, tile);
        const int lo = rg.lo + (k0 << unit_shift), hi = k1 == pl.units ? rg.hi : min(rg.hi, rg.lo + (k1 << unit_shift));
        part = Part{q, pl.s, head, tile, lo, hi, k1 - k0, k1 - k0 == pl.units, u != first};
        if (S) parts = k0 == 0 ? (u + pl.units - 1) / share - (int)blockIdx.x + 1 : 0;
        if (lo < hi) page = (p.b.table + (int64_t)slot_of<S>(p, pl.s) * p.b.max_pages)[min(lo + wave * kBlock + (lane & 31), hi - 1) >> p.c.page_shift];
        // this lane's rows
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
            const int r = tile * R + mt * 16 + col;
            const int i = r / p.group_div, g = r - i * p.group;
            const bool real = r < q.rows * p.group;
            see_hi[mt] = !real ? 0 : p.causal ? min(hi, q.pos0 + i + 1) : hi;
            see_lo[mt] = p.window ? max(lo, q.pos0 + i - p.window + 1) : lo;
            const int at = S ? real ? row_at<S>(p, q, q.row0 + i) : 0 : q.row0 + i;
            const uint16_t *from = p.q + (int64_t)at * p.ldq + (head * p.group + g) * D;
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                const int d = ks * 32 + grp * 8;
                u32x4 x = {0u, 0u, 0u, 0u};
                if (real && d < D) x = ld16<false>(from + d);
                qf[mt][ks] = as_bf16x8(x);
            }
        }
        // tokens that every row of the tile sees; a block that goes beyond them has to be masked
        all_lo = p.window ? q.pos0 + min(q.rows - 1, (tile * R + R - 1) / p.group_div) - p.window + 1 : lo;
        all_hi = p.causal ? min(hi, q.pos0 + tile * R / p.group_div + 1) : hi;
    };
    take(first);
    for (int u = first; u < end;) {
        const int lo = part.lo, hi = part.hi, head = part.head;
        u += part.units;

        f32x4 o[MT][DT];
        float m[MT], l[MT];
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
            m[mt] = -INFINITY;
            l[mt] = 0.f;
#pragma unroll
            for (int d = 0; d < DT; ++d) o[mt][d] = f32x4{0.f, 0.f, 0.f, 0.f};
        }
        const int32_t *table = p.b.table + (int64_t)slot_of<S>(p, part.s) * p.b.max_pages;
        const uint16_t *kbase = p.c.k + head * p.c.head_stride, *vbase = p.c.v + head * p.c.head_stride;

        // lane l looks up the page of the block's token l % 32, a block ahead; tokens past the range are read as
        // its last one and masked below
        unsigned bad = 0;
        for (int j0 = lo + wave * kBlock; j0 < hi; j0 += kWaves * kBlock) {
            bad |= (unsigned)page >= (unsigned)p.c.n_pages;
            const int64_t at = (int64_t)min((unsigned)page, (unsigned)p.c.n_pages - 1u) * p.c.page_stride +
                               (int64_t)(min(j0 + (lane & 31), hi - 1) & place_mask) * p.c.token_stride;
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");       // the block before has been read
            // V is streamed where a tile holds all rows of most sequences, so that nobody reads it again (decode of 256 users
            // 231 -> 214 us, of three long contexts 187 -> 169; K as well 217 and 170: its lines are fetched in two halves);
            // with two tiles of a sequence it costs (drafted rows 38.1 -> 39.1)
#pragma unroll
            for (int k = 0; k < VL; ++k) {
                const int row = k * RPL + lane / CH, d = swizzled<DP>(row, lane % CH) * 8;
                const int64_t from = __shfl(at, row) + d;
                load_to_lds<MT == 1>(FULL || d < D ? (const void *)(vbase + from) : (const void *)zeros, v_lds + k * 1024);
            }
            u32x4 kx[2][KS];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const uint16_t *row = kbase + __shfl(at, h * 16 + col);
#pragma unroll
                for (int ks = 0; ks < KS; ++ks) {
                    const int d = ks * 32 + grp * 8;
                    kx[h][ks] = ld16<false>(row + (FULL ? d : min(d, D - 8)));
                    if (!FULL && d >= D) kx[h][ks] = u32x4{0u, 0u, 0u, 0u};
                }
            }
            page = table[min(j0 + kWaves * kBlock + (lane & 31), hi - 1) >> p.c.page_shift];
            f32x4 sc[MT][2];
#pragma unroll
            for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    sc[mt][h] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int ks = 0; ks < KS; ++ks)
                        sc[mt][h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(kx[h][ks]), qf[mt][ks], sc[mt][h], 0, 0, 0);
                }
            const bool edge = j0 < all_lo || j0 + kBlock > all_hi;
            bf16x8 pf[MT];
            float shrink[MT];
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) {
                float x[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] = sc[mt][e >> 2][e & 3];
                if (edge) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const int j = j0 + (e >> 2) * 16 + grp * 4 + (e & 3);
                        if (j < see_lo[mt] || j >= see_hi[mt]) x[e] = -INFINITY;
                    }
                }
                float top = x[0];
#pragma unroll
                for (int e = 1; e < 8; ++e) top = fmaxf(top, x[e]);
                top = fmaxf(top, __shfl_xor(top, 16));
                top = fmaxf(top, __shfl_xor(top, 32));
                const float now = fmaxf(m[mt], top);
                // the difference is taken before the scale: exact where it matters, however large the scores are
                const float ref = now == -INFINITY ? 0.f : now;
                shrink[mt] = __builtin_amdgcn_exp2f((m[mt] - ref) * p.scale_log2);
                float w[8], sum = 0.f;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    w[e] = __builtin_amdgcn_exp2f((x[e] - ref) * p.scale_log2);
                    sum += w[e];
                }
                l[mt] = l[mt] * shrink[mt] + sum;
                m[mt] = now;
                u32x4 pk;
#pragma unroll
                for (int e = 0; e < 4; ++e) pk[e] = pack_bf16_rne(w[2 * e], w[2 * e + 1]);
                pf[mt] = as_bf16x8(pk);
            }
            wait_loads<0>();
            // V of a token that some rows must not see may be no number: 0 * NaN would reach them
            bool odd = false;
            if (edge) {
#pragma unroll
                for (int d = 0; d < DT; ++d) odd |= not_finite(v_tile<DP>(s_v, d));
                odd = __any(odd);
            }
            if (!odd) {
#pragma unroll
                for (int d = 0; d < DT; ++d) {
                    const bf16x8 v = as_bf16x8(v_tile<DP>(s_v, d));
#pragma unroll
                    for (int mt = 0; mt < MT; ++mt)
                        o[mt][d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, pf[mt], o[mt][d] * shrink[mt], 0, 0, 0);
                }
            } else {
#pragma unroll
                for (int d = 0; d < DT; ++d) {
                    const bf16x8 v = finite_part(as_bf16x8(v_tile<DP>(s_v, d)));
#pragma unroll
                    for (int mt = 0; mt < MT; ++mt)
                        o[mt][d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, pf[mt], o[mt][d] * shrink[mt], 0, 0, 0);
                }
                // the rest is added as it is to the rows that see it.  In blocks without hidden tokens the product does so, but for
                // a weight that has become zero, with which infinity is NaN; so is a sum of infinity that is scaled by zero later
#pragma unroll 1
                for (int j = 0; j < kBlock; ++j)
#pragma unroll
                    for (int d = 0; d < DT; ++d)
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const int c = d * 16 + grp * 4 + e;
                            const float x = odd_part(s_v[j * DP + swizzled<DP>(j, c >> 3) * 8 + (c & 7)]);
#pragma unroll
                            for (int mt = 0; mt < MT; ++mt)
                                if (j0 + j >= see_lo[mt] && j0 + j < see_hi[mt]) o[mt][d][e] += x;
                        }
            }
        }
        if (bad) atomicOr(p.b.status, LORA_STATUS_BAD_PAGE);
        const Part done = part;
        const int begins = parts;
        const int64_t slot = 2 * blockIdx.x + done.later;      // of a part's results: the stretch's first tile, or its last
        if (u < end) take(u);
        // the four waves' parts of the range, 16 rows at a time
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
            float sum_l = l[mt] + __shfl_xor(l[mt], 16);
            sum_l += __shfl_xor(sum_l, 32);
            __syncthreads();
#pragma unroll
            for (int d = 0; d < DT; ++d)
                *reinterpret_cast<f32x4 *>(s_o + (wave * 16 + col) * OS + d * 16 + grp * 4) = o[mt][d];
            if (grp == 0) s_m[wave][col] = m[mt], s_l[wave][col] = sum_l;
            __syncthreads();
            const int row = threadIdx.x >> 4;
            const int r = done.tile * R + mt * 16 + row;
            if (r < done.q.rows * p.group) {
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
                const int i = r / p.group_div;
                int64_t t = done.q.row0 + i;
                const int qh = head * p.group + r - i * p.group;
                int64_t at = slot * R + mt * 16 + row;
                bool final = done.whole;
                float *part_o = p.part_o, *part_ml = p.part_ml;
                if constexpr (S) {            // parts of cut tiles stay, and so does all that is a group's rows'
                    const int64_t group_row = whole_at<S>(p, done.q, done.s, i);
                    t = row_at<S>(p, done.q, done.q.row0 + i);
                    if (begins && group_row >= 0 && (threadIdx.x & 15) == 0) {
                        const int next = (int)((2 * ((int64_t)blockIdx.x + 1)) * R + mt * 16 + row);
                        if (final) note(p, group_row, qh, (int)(group_row * p.heads + qh), 0, 1, kFoundWhole);
                        else note(p, group_row, qh, (int)at, next, begins, kFoundShort);
                    }
                    if (final && group_row >= 0) {
                        at = group_row * p.heads + qh;
                        part_o = p.whole_o;
                        part_ml = p.whole_ml;
                        final = false;
                    }
                }
                const float norm = total == 0.f ? 0.f : 1.f / total;
                for (int d = (threadIdx.x & 15) * 4; d < D; d += 64) {
                    f32x4 sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int w = 0; w < kWaves; ++w)
                        sum += *reinterpret_cast<f32x4 *>(s_o + (w * 16 + row) * OS + d) * f[w];
                    if (final) {
                        u32x2 b;
                        b[0] = pack_bf16_rne(sum[0] * norm, sum[1] * norm);
                        b[1] = pack_bf16_rne(sum[2] * norm, sum[3] * norm);
                        *reinterpret_cast<u32x2 *>(p.out + t * p.ldo + qh * D + d) = b;
                    } else {
                        st16f(part_o + at * D + d, sum);
                    }
                }
                if ((threadIdx.x & 15) == 0) {
                    if (!final) {
                        part_ml[at * 2] = top;
                        part_ml[at * 2 + 1] = total;
                    } else if (p.lse) {
                        p.lse[t * p.heads + qh] = total == 0.f ? -INFINITY : (ref * p.scale_log2 + __builtin_amdgcn_logf(total)) * kLn2;
                    }
                }
            }
        }
        __syncthreads();                 // LDS is V's again
    }
}

// What a row's parts have added up to, by the rule of the running softmax; the sum is that of this lane's set (see join_add).
struct RowSum {
    float m = -INFINITY, total = 0.f;
    f32x4 sum = {0.f, 0.f, 0.f, 0.f};
};

// Adds a row's parts c < n: maximum and sum at ml(c), output at po(c).  Lanes look at 64 parts' maxima and sums at a time, and hand their factors on to the
// lanes that add up the outputs: DP / 4 lanes take one part's 16 bytes each, eight sets of parts are on their way at once.
template <int DP, class Ml, class Out>
__device__ inline void join_add(const AttnParams &p, RowSum &x, int n, Ml ml, Out po)
{
    constexpr int LANES = DP / 4, SETS = 64 / LANES, DEEP = 8;
    const int lane = threadIdx.x & 63, set = lane / LANES, d = (lane % LANES) * 4, D = p.c.dim;
    for (int c0 = 0; c0 < n; c0 += 64) {
        const bool have = c0 + lane < n;
        const float *at = ml(min(c0 + lane, n - 1));
        const float own_m = have ? at[0] : -INFINITY, own_l = have ? at[1] : 0.f;
        float now = own_m;
#pragma unroll
        for (int s = 32; s; s >>= 1) now = fmaxf(now, __shfl_xor(now, s));
        now = fmaxf(x.m, now);
        const float ref = now == -INFINITY ? 0.f : now;
        const float keep = __builtin_amdgcn_exp2f((x.m - ref) * p.scale_log2);
        const float f = __builtin_amdgcn_exp2f((own_m - ref) * p.scale_log2);
        x.total = x.total * keep + last_lane(wave_scan(f * own_l));
        x.sum *= keep;
        x.m = now;
        const int some = min(64, n - c0);
        for (int c = 0; c < some; c += SETS * DEEP) {
            f32x4 o[DEEP];
#pragma unroll
            for (int k = 0; k < DEEP; ++k) {
                const int cc = c + k * SETS + set;
                o[k] = f32x4{0.f, 0.f, 0.f, 0.f};
                if (cc < some && d < D) o[k] = ld16f(po(c0 + cc) + d);
            }
#pragma unroll
            for (int k = 0; k < DEEP; ++k) x.sum += o[k] * __shfl(f, min(c + k * SETS + set, 63));
        }
    }
}

template <int DP>
__device__ inline void join_store(const AttnParams &p, RowSum x, int64_t t, int qh)
{
    constexpr int LANES = DP / 4;
    const int lane = threadIdx.x & 63, set = lane / LANES, d = (lane % LANES) * 4, D = p.c.dim;
#pragma unroll
    for (int s = LANES; s < 64; s <<= 1)
#pragma unroll
        for (int e = 0; e < 4; ++e) x.sum[e] += __shfl_xor(x.sum[e], s);
    const float norm = x.total == 0.f ? 0.f : 1.f / x.total;
    if (set == 0 && d < D) {
        u32x2 b;
        b[0] = pack_bf16_rne(x.sum[0] * norm, x.sum[1] * norm);
        b[1] = pack_bf16_rne(x.sum[2] * norm, x.sum[3] * norm);
        *reinterpret_cast<u32x2 *>(p.out + t * p.ldo + qh * D + d) = b;
    }
    if (lane == 0 && p.lse) {
        const float ref = x.m == -INFINITY ? 0.f : x.m;
        p.lse[t * p.heads + qh] = x.total == 0.f ? -INFINITY : (ref * p.scale_log2 + __builtin_amdgcn_logf(x.total)) * kLn2;
    }
}

// The part of the workgroup b + c of a short tile that begins at unit `start` in workgroup b's stretch: its last tile if it starts
// before, else its first.
__device__ inline int64_t short_part(const AttnParams &p, int b, int c, int start, int share, int row)
{
    return (((int64_t)2 * (b + c) + (c == 0 && start != b * share)) << p.short_shift) + row;
}

// Where the parts of a row of a group and a head are, over the shared tokens or over its own.  Numbers that groups which are not
// true have left are kept in bounds.
struct Found {
    const float *ml, *o;
    int first, second, n, by;
    unsigned room;

    __device__ Found(const AttnParams &p, int4 f)
    {
        const bool is_short = f.w == kFoundShort, is_long = f.w == kFoundLong;
        ml = is_short ? p.part_ml : is_long ? p.long_ml : p.whole_ml;
        o = is_short ? p.part_o : is_long ? p.long_o : p.whole_o;
        room = is_short ? p.parts_short : is_long ? p.parts_long : 2 * p.g.most_rows * p.heads;
        by = is_short ? 2 << p.short_shift : p.c.n_heads * kLongTile;
        n = !room ? 0 : is_short || is_long ? min(max(f.z, 1), 4096) : 1;
        first = f.x;
        second = f.y;
    }

    __device__ int64_t at(int c) const { return min((unsigned)(c == 0 ? first : second + (c - 1) * by), room - 1u); }
};

// Joins the parts of short tiles that lie across the ends of workgroups' stretches: a workgroup per such end, the first
// one inside a tile does it.  Workgroups from join_blocks on, join_long of them: the rows of cut long tiles, a wave per row and head.  Where
// tokens are shared, those behind: the rows of groups, a wave per row and head, over the shared tokens and over their own.
template <int DP, bool S>
__global__ __launch_bounds__(256) void join_kernel(AttnParams p)
{
    const int32_t *plan = p.plan;        // the kernels before have left it
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    // (S: those behind come first, as they have most to do: 61 sequences with drafted rows 42.1 -> 41.7 us, 32 answers 22.0 -> 21.1)
    const int others = p.join_blocks + p.join_long, found = gridDim.x - others;
    const int id = !S ? blockIdx.x : (int)blockIdx.x < found ? blockIdx.x + others : blockIdx.x - found;
    if (id < p.join_blocks) {
        const int share = uniform(plan[kShare]), b = id, cut = (b + 1) * share;
        if (cut >= plan[kUnits]) return;
        Seq<S> q;
        const Place pl = place_of<S>(p, plan, cut, q);
        if (pl.start == cut || pl.start < b * share) return;       // between two tiles, or not the first end inside this one
        if (S && whole_at<S>(p, q, pl.s, 0) >= 0) return;          // of a group
        const int n = (pl.start + pl.units - 1) / share - b + 1;
        const int rows = min(1 << p.short_shift, q.rows * p.group - (pl.tile << p.short_shift));
        for (int row = blockIdx.y * 4 + wave; row < rows; row += 4 * gridDim.y) {
            const int r = (pl.tile << p.short_shift) + row, i = r / p.group_div;
            RowSum x;
            const auto part = [&](int c) { return short_part(p, b, c, pl.start, share, row); };
            join_add<DP>(p, x, n, [&](int c) { return p.part_ml + part(c) * 2; }, [&](int c) { return p.part_o + part(c) * p.c.dim; });
            join_store<DP>(p, x, q.row0 + i, pl.head * p.group + r - i * p.group);
        }
        return;
    }
    if (blockIdx.y) return;
    const int seqs = plan_seqs<S>(p), block = id - p.join_blocks;
    if (S && block >= p.join_long) {
        const int n = plan[kGroupRows] * p.heads;
        for (int u = (block - p.join_long) * 4 + wave; u < n; u += found * 4) {
            const Found a(p, p.found[u]), b(p, p.found[u + p.g.most_rows * p.heads]);
            const int v = u / p.heads_div, t = min((unsigned)p.g.rows[v], (unsigned)p.b.n_rows - 1u);
            RowSum x;
            join_add<DP>(p, x, a.n + b.n, [&](int c) { return c < a.n ? a.ml + a.at(c) * 2 : b.ml + b.at(c - a.n) * 2; },
                         [&](int c) { return c < a.n ? a.o + a.at(c) * p.c.dim : b.o + b.at(c - a.n) * p.c.dim; });
            join_store<DP>(p, x, t, u - v * p.heads);
        }
        return;
    }
    const int32_t *base = plan + kPlanHead + kBaseJoin * seqs, *slots = plan + kPlanHead + kBaseSlot * seqs;
    const int units = plan[kJoinUnits], chunk = plan[kChunk];
    for (int u = block * 4 + wave; u < units; u += p.join_long * 4) {
        const int s = seq_at<S>(p, base, u);
        const Seq<S> q = planned_seq<S>(p, plan, s);
        const int left = u - base[s];
        const int i = left / p.heads_div, qh = left - i * p.heads;
        const int head = qh / p.group_div;
        const int r = i * p.group + qh - head * p.group, tile = r / kLongTile;
        const Range rg = range_of<kLong>(p, q, tile);
        const int cuts = splits_of(rg.hi - rg.lo, chunk);
        if (cuts == 1 || (S && whole_at<S>(p, q, s, i) >= 0)) continue;
        const int slot = slots[s] + tile * splits_of(reach_of<kLong>(p, q), chunk) * p.c.n_heads + head;
        RowSum x;
        const auto part = [&](int c) { return (int64_t)(slot + c * p.c.n_heads) * kLongTile + r - tile * kLongTile; };
        join_add<DP>(p, x, cuts, [&](int c) { return p.long_ml + part(c) * 2; }, [&](int c) { return p.long_o + part(c) * p.c.dim; });
        join_store<DP>(p, x, q.row0 + i, qh);
    }
}

template <int DP, int MT, int BLOCKS, bool S>
void launch_attend(const AttnParams &p, unsigned grid, hipStream_t s)
{
    if (p.c.dim == DP) hipLaunchKernelGGL((attend_kernel<DP, MT, true, BLOCKS, S>), dim3(grid), dim3(kWaves * 64), 0, s, p);
    else hipLaunchKernelGGL((attend_kernel<DP, MT, false, BLOCKS, S>), dim3(grid), dim3(kWaves * 64), 0, s, p);
}

// Where the workspace has what, and which kernels run.
void lay_out(AttnParams &p, const Kinds &k, const AttnWs &at, void *ws)
{
    char *w = static_cast<char *>(ws);
    p.plan = reinterpret_cast<int32_t *>(w + at.plan);
    p.part_ml = reinterpret_cast<float *>(w + at.short_ml);
    p.part_o = reinterpret_cast<float *>(w + at.short_o);
    p.long_ml = reinterpret_cast<float *>(w + at.long_ml);
    p.long_o = k.has_long ? reinterpret_cast<float *>(w + at.long_o) : nullptr;
    p.short_limit = k.limit;
    p.short_shift = k.shift;
    p.short_blocks = k.blocks;
}

// The kernel of short tiles, `tiles` of a head at most; its workgroups.
template <bool S>
unsigned launch_short(const AttnParams &p, const Kinds &k, int64_t reach, int64_t tiles, hipStream_t s)
{
    unsigned grid = 0;
    if (k.has_short) {
        grid = (unsigned)std::min<int64_t>(k.blocks, tiles * p.c.n_heads * ((reach + (1 << kUnitShift) - 1) >> kUnitShift));
        if (p.c.dim <= 64 && k.shift == 5) launch_attend<64, 2, 2, S>(p, grid, s);
        else if (p.c.dim <= 64) launch_attend<64, 1, 3, S>(p, grid, s);
        else if (p.c.dim <= 128 && k.shift == 5) launch_attend<128, 2, 2, S>(p, grid, s);
        else if (p.c.dim <= 128) launch_attend<128, 1, 3, S>(p, grid, s);
        else launch_attend<256, 1, 2, S>(p, grid, s);
    }
    return grid;
}

// The join of the short tiles' parts that `grid` workgroups have left, and of the long tiles'.  join_rows: rows of a tile that
// join_kernel takes side by side; shared: workgroups for the rows of groups.
template <bool S>
hipError_t launch_join(AttnParams &p, const Kinds &k, int64_t reach, unsigned grid, unsigned join_rows, unsigned shared, hipStream_t s)
{
    // parts: of short tiles of more than one unit, of long ones that may be cut
    p.join_long = k.has_long && reach > kLongMinSplit ? 1024 : 0;
    p.join_blocks = k.has_short && reach > 1 << kUnitShift ? (int)grid - 1 : 0;
    if (p.join_blocks + p.join_long + shared > 0) {
        const dim3 both(p.join_blocks + p.join_long + shared, (join_rows + 3) / 4), block(256);
        if (p.c.dim <= 64) hipLaunchKernelGGL((join_kernel<64, S>), both, block, 0, s, p);
        else if (p.c.dim <= 128) hipLaunchKernelGGL((join_kernel<128, S>), both, block, 0, s, p);
        else hipLaunchKernelGGL((join_kernel<256, S>), both, block, 0, s, p);
    }
    return hipGetLastError();
}

struct SharedWs : AttnWs {
    size_t whole_ml, whole_o, found;
};

SharedWs shared_ws_of(int n_seqs, int group_rows, const SharedKinds &k, int heads, int dim)
{
    SharedWs w;
    static_cast<AttnWs &>(w) = attn_ws_of(groups_of(n_seqs) + n_seqs, k, dim, kSharedArrays, kSharedTarget);
    const size_t rows = 2 * (size_t)group_rows * heads;
    w.whole_ml = w.bytes;
    w.whole_o = w.whole_ml + up256(rows * 8);
    w.found = w.whole_o + up256(rows * dim * 4);
    w.bytes = w.found + up256(rows * sizeof(int4));
    return w;
}

}  // namespace

size_t attention_ws_bytes(int n_seqs, int n_rows, int max_rows, int heads, int kv_heads, int dim)
{
    return attn_ws_of(n_seqs, kinds_of(n_seqs, n_rows, max_rows, heads, kv_heads, dim), dim).bytes;
}

hipError_t launch_attention(AttnParams &p, int max_rows, void *ws, hipStream_t s)
{
    const Kinds k = kinds_of(p.b.n_seqs, p.b.n_rows, max_rows, p.heads, p.c.n_heads, p.c.dim);
    lay_out(p, k, attn_ws_of(p.b.n_seqs, k, p.c.dim), ws);
    if (p.b.n_seqs > kInlineSeqs) hipLaunchKernelGGL(plan_kernel<false>, dim3(1), dim3(kPlanThreads), 0, s, p);
    if (k.has_long) {
        const hipError_t e = launch_attend_long(p, (int)k.long_items, s);
        if (e != hipSuccess) return e;
    }
    const int64_t reach = p.window ? std::min<int64_t>(p.b.tokens_max, (int64_t)p.window + kLongTile) : p.b.tokens_max;
    const int64_t tiles = std::min(p.b.n_seqs, p.b.n_rows) + ((int64_t)p.b.n_rows * p.group >> k.shift);
    // a wave per row of a tile, or per four rows where most sequences are likely to have one new row only
    const unsigned rows = k.has_long ? 1 : (unsigned)std::min<int64_t>(1 << k.shift, (int64_t)(max_rows > 0 ? max_rows : p.b.n_rows) * p.group);
    return launch_join<false>(p, k, reach, launch_short<false>(p, k, reach, tiles, s), rows, 0, s);
}

size_t attention_shared_ws_bytes(int n_seqs, int n_rows, int max_rows, int group_rows, int max_group_rows, int heads, int kv_heads, int dim)
{
    const SharedKinds k = shared_kinds_of(n_seqs, n_rows, max_rows, group_rows, max_group_rows, heads, kv_heads, dim);
    return shared_ws_of(n_seqs, group_rows, k, heads, dim).bytes;
}

hipError_t launch_attention_shared(AttnParams &p, int max_rows, int max_group_rows, void *ws, hipStream_t s)
{
    const SharedKinds k = shared_kinds_of(p.b.n_seqs, p.b.n_rows, max_rows, p.g.most_rows, max_group_rows, p.heads, p.c.n_heads, p.c.dim);
    const SharedWs at = shared_ws_of(p.b.n_seqs, p.g.most_rows, k, p.heads, p.c.dim);
    lay_out(p, k, at, ws);
    p.group_limit = k.group_limit;
    p.whole_ml = reinterpret_cast<float *>(static_cast<char *>(ws) + at.whole_ml);
    p.whole_o = reinterpret_cast<float *>(static_cast<char *>(ws) + at.whole_o);
    p.found = reinterpret_cast<int4 *>(static_cast<char *>(ws) + at.found);
    p.parts_short = 2 * k.blocks << k.shift;
    p.parts_long = k.has_long ? 2 * kSharedTarget * kLongTile : 0;
    if (p.g.most + p.b.n_seqs > kSharedInline) hipLaunchKernelGGL(plan_kernel<true>, dim3(1), dim3(kPlanThreads), 0, s, p);
    const int64_t rows = (int64_t)p.b.n_rows + p.g.most_rows;
    const int64_t tiles = std::min(p.b.n_seqs, p.b.n_rows) + p.g.most + (rows * p.group >> k.shift);
    const unsigned shared = (unsigned)std::min<int64_t>(((int64_t)p.g.most_rows * p.heads + 3) / 4, 8192);
    // the short tiles' kernel first: it leaves a plan that it has made to the long ones', which so has little to do where there are none
    const unsigned grid = launch_short<true>(p, k, p.b.tokens_max, tiles, s);
    if (k.has_long) {
        const hipError_t e = launch_attend_long_shared(p, (int)k.long_items, s);
        if (e != hipSuccess) return e;
    }
    // most tiles are of groups or of sequences in one, and the workgroups behind join them
    return launch_join<true>(p, k, p.b.tokens_max, grid, 4, shared, s);
}

}  // namespace lora
