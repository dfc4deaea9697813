// Attention of long chunks of new rows over the paged cache: tiles of 128 rows, four waves of 32 rows each.
//
// K and V of 64 tokens at a time go straight into LDS, where all waves read them, while the 64 before are
// worked on.  S^T = K Q^T and O^T = V^T P^T on v_mfma_f32_32x32x16_bf16, as in kv_attention.hip: a lane's column is one row
// of the tile, its two lane halves hold different tokens, and P goes from the first product's result to the second
// one's operand without leaving its lane (16 tokens: 4 h .. 4 h + 3 and 8 + 4 h .. 8 + 4 h + 3 for lane half h).  The weights are
// rounded to bf16 for it as there: 2^-8 of each at most; their sum takes them unrounded.
//
// Weights need not be taken against the running maximum, only against a value near it: the reference is the maximum of the
// first tokens that a row sees, and moves to the running one when the weights of a step pass 2^10.  So most steps look for
// no maximum and rescale nothing; the sums are the same up to rounding.
//
// Measured, 32 / 8 heads of 128: 8 prompts of 2048 rows 357 us, 770 TFLOP/s of the visible pairs; 1984 rows over 18000 tokens 585 us,
// 930 TFLOP/s (a large library product reaches 1369 TFLOP/s on this card).  That is once the clock has settled under such work: the first twenty
// launches after idling take 394 - 490 and 615 - 719 us.  Of the SIMDs' time in the second the products take 44 % and vector instructions
// 53 %: of about 250 per step 117 form the weights, 64 copy the outputs' registers around the product with V, 48 form addresses
// of loads.  LDS is busy for 66 % (K 8 cycles a read of 1 KiB, V 8 cycles a transposed read of 512 bytes).
// Tried and left out, as slower: 64 rows per wave, which halves the LDS reads but needs 512 registers, between whose two
// halves the compiler moves the outputs at every branch (2.2 ms; 377 us with 32); a step's scores formed while the weights of
// the step before are (spills, 564 us), or its products of both kinds in one stretch (453 us); eight waves on K and V (a batch
// with the 1984 rows 744 us against 771, but 7 to 21 % slower below 2000 tokens).
#include <type_traits>

#include "kv_attention.h"

namespace lora {

namespace {

constexpr int kRows = kLongTile;
constexpr int kTokens = 64;              // of a step
constexpr int kWaves = 4;
constexpr float kMost = 1024.f;          // sum of a lane's 32 weights up to which the reference stays
constexpr float kExact = 4096.f;         // scaled maxima up to which e^(s - m) is formed with one rounding of m

typedef __attribute__((ext_vector_type(16))) float f32x16;

__device__ __align__(16) const unsigned zeros[4] = {0u, 0u, 0u, 0u};

typedef __attribute__((address_space(3))) const u32x4 lds_u32x4;
typedef __attribute__((ext_vector_type(4))) short s16x4;
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
typedef __attribute__((address_space(3))) const uint16_t lds_u16;
typedef __attribute__((address_space(3))) unsigned char lds_byte;

__device__ inline float other_half(float x) { return __shfl_xor(x, 32); }

// The value of the lane of the same DP / 8 lanes that holds load j's row.
template <int DP>
__device__ inline int of_load(int x, int j)
{
    if (DP == 64) return __shfl(x, (threadIdx.x & 56) + j);
    switch (j) {                          // row_newbcast: one lane of each 16
    case 0: return __builtin_amdgcn_update_dpp(0, x, 0x150, 0xf, 0xf, true);
    case 1: return __builtin_amdgcn_update_dpp(0, x, 0x151, 0xf, 0xf, true);
    case 2: return __builtin_amdgcn_update_dpp(0, x, 0x152, 0xf, 0xf, true);
    case 3: return __builtin_amdgcn_update_dpp(0, x, 0x153, 0xf, 0xf, true);
    case 4: return __builtin_amdgcn_update_dpp(0, x, 0x154, 0xf, 0xf, true);
    case 5: return __builtin_amdgcn_update_dpp(0, x, 0x155, 0xf, 0xf, true);
    case 6: return __builtin_amdgcn_update_dpp(0, x, 0x156, 0xf, 0xf, true);
    default: return __builtin_amdgcn_update_dpp(0, x, 0x157, 0xf, 0xf, true);
    }
}

// DP: width of a head rounded up.  FULL: it is the width itself; otherwise pieces beyond it are filled with zeros.
// S: sequences share tokens.
template <int DP, bool FULL, bool S>
__global__ __launch_bounds__(kWaves * 64, DP > 128 ? 1 : 2) void attend_long_kernel(AttnParams p)
{
    constexpr int KS = DP / 16;          // steps of the first product
    constexpr int DT = DP / 32;          // output tiles of the second
    constexpr int CH = DP / 8;           // 16-byte pieces of a row
    constexpr int RPL = 64 / CH;         // rows that a wave's load covers
    constexpr int NL = kTokens / RPL / kWaves;           // loads of K and of V per wave and step
    constexpr int ROW = DP * 2;          // bytes
    constexpr int STAGE = kTokens * ROW; // of K or V in LDS
    __shared__ __align__(16) unsigned char s_kv[2][2][STAGE];

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int col = lane & 31, half = lane >> 5;
    const int D = FULL ? DP : p.c.dim;
    __shared__ int32_t s_plan[S ? 1 : kInlineWords<S>];
    // (S: the kernels before have left it)
    const int32_t *plan = S ? p.plan : plan_of<S>(p, s_plan);
    const int n = blockIdx.x;
    if (n >= plan[kItems]) return;
    // the cuts of a tile lie n_heads apart, tiles behind each other, those with the longest ranges first
    const int32_t *base = plan + kPlanHead + kBaseItem * plan_seqs<S>(p);
    const int seq = seq_at<S>(p, base, n);
    const Seq<S> q = planned_seq<S>(p, plan, seq);
    const int left = uniform(n - base[seq]);
    const int pair = left / p.kv_div, head = left - pair * p.c.n_heads;
    const int chunk = uniform(plan[kChunk]);
    const int cuts = splits_of(reach_of<kLong>(p, q), chunk);
    const int turn_no = cuts == 1 ? pair : pair / cuts, cut = pair - turn_no * cuts;
    const int tile = tiles_of<kLong>(p, q, S ? uniform(plan[kGroupLimit]) : 0) - 1 - turn_no;
    const Range rg = range_of<kLong>(p, q, tile);
    const int splits = splits_of(rg.hi - rg.lo, chunk);
    if (cut >= splits) return;
    const int each = cut_of(rg, splits);
    const int lo = rg.lo + cut * each, hi = min(rg.hi, lo + each);
    const int slot = plan[kPlanHead + kBaseSlot * plan_seqs<S>(p) + seq] + (tile * cuts + cut) * p.c.n_heads + head;

    // this lane's row, and the tokens that it, some row and every row of its wave see
    const int r0 = tile * kRows + wave * 32;
    const int n_rows = q.rows * p.group;
    const int r = r0 + col;
    const int i = r / p.group_div, g = r - i * p.group;
    const bool real = r < n_rows;
    const int64_t t = S ? real ? row_at<S>(p, q, q.row0 + i) : 0 : q.row0 + i;
    const int qh = head * p.group + g;
    const int see_hi = !real ? 0 : p.causal ? min(hi, q.pos0 + i + 1) : hi;
    const int see_lo = p.window ? max(lo, q.pos0 + i - p.window + 1) : lo;
    const int first_i = r0 / p.group_div, last_i = min(q.rows - 1, (r0 + 31) / p.group_div);
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
    // The reference m that weights are taken against (of a row that has seen nothing: none), the same in powers of two,
    // and this lane's part of the sum.  A row beyond the tile's takes zero, so that it never asks for another.
    float m = real ? -INFINITY : 0.f, ms = m, l = 0.f;
    bool big = false;

    // LDS addresses of the operands: only constants are added to them in the loop
    lds_byte *const lds0 = (lds_byte *)&s_kv[0][0][0];
    lds_byte *k_at[KS], *v_at[DT];
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) k_at[ks] = lds0 + col * ROW + swizzled<DP>(col, ks * 2 + half) * 16;
    {
        const int l16 = lane & 15, grp = lane >> 4, row = (grp >> 1) * 4 + (l16 >> 2);
#pragma unroll
        for (int d = 0; d < DT; ++d)
            v_at[d] = lds0 + STAGE + row * ROW + swizzled<DP>(row, d * 4 + (grp & 1) * 2 + (l16 >> 1 & 1)) * 16 + (l16 & 1) * 8;
    }

    // This wave's loads of a step: load j covers rows (wave * NL + j) * RPL + lane / CH.  Lane j of every CH lanes looks up
    // the page of load j's row and hands the place to the others; a lane fetches the piece that belongs at its place.
    const int32_t *table = p.b.table + (int64_t)slot_of<S>(p, seq) * p.b.max_pages;
    const int place_mask = (1 << p.c.page_shift) - 1;
    const uint16_t *kbase = p.c.k + head * p.c.head_stride, *vbase = p.c.v + head * p.c.head_stride;
    const int my_row = (wave * NL + (lane & (NL - 1))) * RPL + lane / CH;
    int piece[2];                         // of even and of odd loads
#pragma unroll
    for (int j = 0; j < 2; ++j) piece[j] = swizzled<DP>((wave * NL + j) * RPL + lane / CH, lane % CH) * 8;
    static_assert(RPL * 2 >= 8 || DP > 128, "the swizzle repeats after two loads");
    int page = 0;
    unsigned bad = 0;
    const auto fetch_page = [&](int j0) { page = table[min(j0 + my_row, hi - 1) >> p.c.page_shift]; };
    const auto fetch = [&](int j0, int stage) {
        bad |= (unsigned)page >= (unsigned)p.c.n_pages;
        const int64_t at = (int64_t)min((unsigned)page, (unsigned)p.c.n_pages - 1u) * p.c.page_stride +
                           (int64_t)(min(j0 + my_row, hi - 1) & place_mask) * p.c.token_stride;
        const int at_lo = (int)at, at_hi = (int)(at >> 32);
#pragma unroll
        for (int j = 0; j < NL; ++j) {
            const int64_t row = (int64_t)(((uint64_t)(unsigned)of_load<DP>(at_hi, j) << 32) | (unsigned)of_load<DP>(at_lo, j));
            const int pc = DP > 128 ? swizzled<DP>((wave * NL + j) * RPL + lane / CH, lane % CH) * 8 : piece[j & 1];
            const bool in = FULL || pc < D;
            const unsigned to = (unsigned)(uintptr_t)lds0 + stage * 2 * STAGE + (wave * NL + j) * 1024;
            load_to_lds<false>(in ? (const void *)(kbase + row + pc) : (const void *)zeros, to);
            load_to_lds<false>(in ? (const void *)(vbase + row + pc) : (const void *)zeros, to + STAGE);
        }
    };

    // 64 tokens from j0 on, in LDS at `stage`
    const auto step = [&](int j0, auto stage_c) {
        constexpr int AT = decltype(stage_c)::value * 2 * STAGE;
        const auto v_tile = [&](int k, int d) {
            const u32x2 a = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(v_at[d] + (AT + k * 16 * ROW))));
            const u32x2 b = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(v_at[d] + (AT + k * 16 * ROW + 8 * ROW))));
            return as_bf16x8(u32x4{a[0], a[1], b[0], b[1]});
        };
        f32x16 s[2] = {f32x16{}, f32x16{}};
        __builtin_amdgcn_s_setprio(1);       // the wave beside this one forms weights meanwhile, or waits
#pragma unroll
        for (int ks = 0; ks < KS; ++ks)
#pragma unroll
            for (int h = 0; h < 2; ++h)
                s[h] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(*(lds_u32x4 *)(k_at[ks] + (AT + h * 32 * ROW))), qf[ks], s[h], 0, 0, 0);
        // six operands are on their way ahead of the products
        __builtin_amdgcn_sched_group_barrier(0x100, 6, 0);
#pragma unroll
        for (int k = 0; k < KS * 2 - 6; ++k) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
        }
        __builtin_amdgcn_sched_group_barrier(0x008, 6, 0);
        __builtin_amdgcn_s_setprio(0);
        const bool edge = j0 < all_lo || j0 + kTokens > all_hi;
        if (edge) {
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    if ((unsigned)(j0 + 4 * half - see_lo + h * 32 + 8 * (e >> 2) + (e & 3)) >= (unsigned)max(0, see_hi - see_lo)) s[h][e] = -INFINITY;
        }
        bf16x8 pf[4];
        float sum;
        const auto weigh = [&](float mul, float sub) {
            sum = 0.f;
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
        };
        bool again = big;
        if (!big) {
            weigh(p.scale_log2, ms == -INFINITY ? 0.f : ms);
            again = __any(sum > kMost || ms == -INFINITY);
        }
        if (again) {
            float top = s[0][0];
#pragma unroll
            for (int e = 1; e < 32; ++e) top = fmaxf(top, s[e >> 4][e & 15]);
            top = fmaxf(top, other_half(top));
            const float now = fmaxf(m, top), now_s = fmaxf(ms, top * p.scale_log2);
            const bool was_big = big;
            big = __any(fabsf(now_s) > kExact && now > -INFINITY);
            const float ref = now == -INFINITY ? 0.f : now;
            // scores so large that m's own rounding in powers of two would show are subtracted before they are scaled
            const float keep = now == -INFINITY ? 1.f
                               : was_big || big ? __builtin_amdgcn_exp2f((m - ref) * p.scale_log2)
                                                : __builtin_amdgcn_exp2f(ms - now_s);
            l *= keep;
#pragma unroll
            for (int d = 0; d < DT; ++d) o[d] *= keep;
            m = now;
            ms = now_s;
            if (big) {
#pragma unroll
                for (int e = 0; e < 32; ++e) s[e >> 4][e & 15] = (s[e >> 4][e & 15] - ref) * p.scale_log2;
                weigh(1.f, 0.f);
            } else {
                weigh(p.scale_log2, now_s == -INFINITY ? 0.f : now_s);
            }
        }
        l += sum;
        // V of a token that some rows must not see may be no number: 0 * NaN would reach them
        bool odd = false;
        if (edge) {
#pragma unroll
            for (int k = 0; k < 4; ++k)
#pragma unroll
                for (int d = 0; d < DT; ++d) odd |= not_finite(__builtin_bit_cast(u32x4, v_tile(k, d)));
            odd = __any(odd);
        }
        if (!odd) {
            __builtin_amdgcn_s_setprio(1);
#pragma unroll
            for (int k = 0; k < 4; ++k)
#pragma unroll
                for (int d = 0; d < DT; ++d) o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v_tile(k, d), pf[k], o[d], 0, 0, 0);
            __builtin_amdgcn_sched_group_barrier(0x100, 8, 0);
#pragma unroll
            for (int k = 0; k < 4 * DT - 4; ++k) {
                __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
            }
            __builtin_amdgcn_sched_group_barrier(0x008, 4, 0);
            __builtin_amdgcn_s_setprio(0);
        } else {
#pragma unroll
            for (int k = 0; k < 4; ++k)
#pragma unroll
                for (int d = 0; d < DT; ++d)
                    o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(finite_part(v_tile(k, d)), pf[k], o[d], 0, 0, 0);
            // the rest is added as it is to the rows that see it.  In steps without hidden tokens the product does so, but for a
            // weight that has become zero, with which infinity is NaN; so is a sum of infinity that is scaled by zero later
#pragma unroll 1
            for (int j = 0; j < kTokens; ++j) {
                if (j0 + j < see_lo || j0 + j >= see_hi) continue;
#pragma unroll
                for (int d = 0; d < DT; ++d)
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        const int c = d * 32 + 8 * (e >> 2) + 4 * half + (e & 3);
                        o[d][e] += odd_part(*(lds_u16 *)(lds0 + AT + STAGE + j * ROW + swizzled<DP>(j, c >> 3) * 16 + (c & 7) * 2));
                    }
            }
        }
    };
    // the stage is full, and every wave has read what the next fetch overwrites
    const auto meet = [&] {
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_waitcnt(0x0070);            // vmcnt(0) lgkmcnt(0); the loads into LDS count as well
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };
    const auto turn = [&](int j0, auto stage_c) {
        meet();
        if (j0 + kTokens < hi) {
            fetch(j0 + kTokens, decltype(stage_c)::value ^ 1);
            fetch_page(j0 + 2 * kTokens);
        }
        if (j0 < any_hi && j0 + kTokens > any_lo) step(j0, stage_c);
    };
    if (lo < hi) {
        fetch_page(lo);
        fetch(lo, 0);
        fetch_page(lo + kTokens);
    }
    for (int j0 = lo; j0 < hi; j0 += 2 * kTokens) {
        turn(j0, std::integral_constant<int, 0>{});
        if (j0 + kTokens < hi) turn(j0 + kTokens, std::integral_constant<int, 1>{});
    }
    if (bad) atomicOr(p.b.status, LORA_STATUS_BAD_PAGE);
    l += other_half(l);
    if (!real) return;
    const float ref = ms == -INFINITY ? 0.f : ms;
    const int64_t group_row = whole_at<S>(p, q, seq, i), whole = splits == 1 ? group_row : -1;
    if (splits == 1 && whole < 0) {
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
        const int64_t at = whole < 0 ? (int64_t)slot * kRows + wave * 32 + col : whole * p.heads + qh;
        float *part_o = whole < 0 ? p.long_o : p.whole_o, *part_ml = whole < 0 ? p.long_ml : p.whole_ml;
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int c = d * 32 + e * 8 + half * 4;
                if (c < D) st16f(part_o + at * D + c, f32x4{o[d][4 * e], o[d][4 * e + 1], o[d][4 * e + 2], o[d][4 * e + 3]});
            }
        if (half == 0) {
            if (S && cut == 0 && group_row >= 0)
                note(p, group_row, qh, (int)at, (int)at + p.c.n_heads * kRows, splits, whole < 0 ? kFoundLong : kFoundWhole);
            part_ml[at * 2] = m;
            part_ml[at * 2 + 1] = l;
        }
    }
}

}  // namespace

namespace {

template <bool S>
hipError_t launch_long(const AttnParams &p, int max_items, hipStream_t s)
{
    const dim3 grid(max_items), block(kWaves * 64);
#define LORA_LONG(DP)                                                                                          \
    if (p.c.dim == DP) hipLaunchKernelGGL((attend_long_kernel<DP, true, S>), grid, block, 0, s, p);            \
    else if (p.c.dim < DP) hipLaunchKernelGGL((attend_long_kernel<DP, false, S>), grid, block, 0, s, p);
    if (p.c.dim <= 64) {
        LORA_LONG(64)
    } else if (p.c.dim <= 128) {
        LORA_LONG(128)
    } else {
        LORA_LONG(256)
    }
#undef LORA_LONG
    return hipGetLastError();
}

}  // namespace

hipError_t launch_attend_long(const AttnParams &p, int max_items, hipStream_t s) { return launch_long<false>(p, max_items, s); }
hipError_t launch_attend_long_shared(const AttnParams &p, int max_items, hipStream_t s) { return launch_long<true>(p, max_items, s); }

}  // namespace lora
