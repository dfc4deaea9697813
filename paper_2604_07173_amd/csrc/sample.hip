// The next token of a row of logits: a workgroup per row, which goes through it two to four times.
//
// All limits cut the order of falling logits (equal ones by number), so what is kept is its beginning: the tokens above a border
// value and the first few, by number, of those that are equal to it.  No sort is needed for that:
//   1  the largest logit
//   2  the border of top_k.  Where k of the threads' largest logits lie above a value, so do the k first tokens: what is above it is
//      listed in LDS.  A short list settles everything by comparing its tokens in pairs: their places in the order, the weights before
//      them there, and the kept weights before them by number
//   3  otherwise the tokens are counted in bins of falling logits, those of the border's bin are listed and counted in bins of their bits, finer
//      each time, until one value is left (and all above it, if they fit); and the border of top_p in the same way, with weights instead of numbers.  The weights' bins
//      are kept for each wave's stretch of the vocabulary apart, so that with the border its kept weight is known as well
//   4  the stretch in which u is reached is divided among the waves again, and the last wave goes through a few steps of 64 lanes'
//      logits.  How many of the border's value are kept is counted along
//
// A weight is 2^x, x = (l - max) log2(e) / T, formed in 64 bits from a table of 2^(j/1024) and a polynomial of 2^(f/1024), |f| <= 1/2, whose
// cubic term (below 2^-37) is put into the linear one, which leaves a quarter of it; and taken as a whole multiple of 2^-shift: the sums
// of whole numbers are exact, so threads may add them in any order.  The order of tokens is that of the logits' bits.
//
// Bound by the instructions that form weights, 24 for each token that has one, four cycles a wave at 64 bits (28 us for 128000 tokens of a
// row), and by the latency of a pass and of its sums over the workgroup, some 3 us each; the reading comes third.  64 rows of
// 128000 fp32 logits (33 MB) with limits of their own 82 to 113 us, 512 of 50257 bf16 (51 MB) with top_p = 0.95 69 us, one of 32000 with top_k = 50 and
// top_p = 0.9 12.5 us, of which a launch takes 3.
#include <limits.h>

#include <algorithm>
#include <type_traits>

#include "kv_device.h"
#include "sample_bins.h"
#include "step_internal.h"

namespace lora {

namespace {

typedef unsigned long long u64;

constexpr int kTable = 1024;
// Rows up to which each has a CU to itself, whose waves all work on it; more share CUs, in workgroups of half as many.  Small vocabularies
// take fewer threads, so that barriers and sums over the workgroup cost less.  us with top_p = 0.95, 1024 / 512 / 256 threads:
//   256 rows of 64000 fp32     60.1 /  62.1 /  99      512 rows of 128000 bf16   154.2 / 135.6 / 501
//   64 of 200000              107.3 / 142.0 / 854      1024 of 64000             186.0 / 141.9 / 147
//   1 of 32000                 30.6 /  32.3 /  47      64 of 2000                 21.1 /  16.8 /  15.7
// and with limits that differ from row to row (300 rows of 64000, few of which take long: 64 / 78)
//   64 of 16000                39.7 /  38.8 /  52      1 of 4000                  25.6 /  17.1 /  17.7
//   64 of 8192                 35.2 /  29.0 /  34.8    64 of 1000                 28.6 /  22.0 /  20.3
//   1024 of 8000               90.7 /  49.9 /  43.0    1024 of 32000             122.2 /  81.4 /  90.6
constexpr int kRowsAlone = 256, kSmallVocab = 16384, kTinyVocab = 2048, kTinyVocabMany = 8192;
// Of a row's tokens, the part at most that is listed whole
constexpr int kListedOf = 4;
constexpr double kMagic = 4503599627370496.0;      // 2^52: added to a number below it, leaves its rounding to a whole one in the low bits

// The order of floats as that of whole numbers; -0 and 0 are one value.
__device__ inline unsigned key_of(float l)
{
    const unsigned b = __float_as_uint(l + 0.f);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}

__device__ inline float of_key(unsigned k) { return __uint_as_float(k & 0x80000000u ? k & 0x7FFFFFFFu : ~k); }

// A row as 16-byte pieces of memory, four or eight logits each.
template <bool F32>
struct Row : Pieces<F32 ? 4 : 8> {
    static constexpr int VEC = F32 ? 4 : 8, SIZE = F32 ? 4 : 2;
    using Pieces<VEC>::skew;
    using Pieces<VEC>::vocab;
    const char *base;

    __device__ Row(const void *logits, int64_t at, int vocab)
    {
        const uintptr_t first = reinterpret_cast<uintptr_t>(logits) + at * SIZE;
        base = reinterpret_cast<const char *>(first & ~(uintptr_t)15);
        this->skew = (int)(first & 15) / SIZE;
        this->vocab = vocab;
    }

    // Piece i; -inf, which is never chosen, in place of what is not the row's.
    __device__ u32x4 load(int i) const
    {
        constexpr unsigned none = F32 ? 0xFF800000u : 0xFF80FF80u;
        u32x4 v = {none, none, none, none};
        const int first = i * VEC - skew;
        if (first >= 0 && first + VEC <= vocab) {
            v = ld16<false>(base + (int64_t)i * 16);
        } else if (first < vocab) {
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                if (first + e < 0 || first + e >= vocab) continue;
                if (F32) {
                    v[e & 3] = *(const LORA_GLOBAL unsigned *)(base + (int64_t)i * 16 + e * 4);
                } else {
                    const unsigned x = *(const LORA_GLOBAL uint16_t *)(base + (int64_t)i * 16 + e * 2);
                    v[e >> 1] = e & 1 ? (v[e >> 1] & 0xFFFFu) | x << 16 : (v[e >> 1] & 0xFFFF0000u) | x;
                }
            }
        }
        return v;
    }

    // Logit i of the row.
    __device__ float one(int i) const
    {
        const char *at = base + ((int64_t)skew + i) * SIZE;
        return __uint_as_float(F32 ? *(const LORA_GLOBAL unsigned *)at : (unsigned)*(const LORA_GLOBAL uint16_t *)at << 16);
    }

    // Logit e of a piece.
    static __device__ float at(u32x4 v, int e)
    {
        return F32 ? __uint_as_float(v[e & 3]) : __uint_as_float(e & 1 ? v[e >> 1] & 0xFFFF0000u : v[e >> 1] << 16);
    }
};

// What a row's weights are formed with.
struct Weigh {
    const double *table;                  // 2^(j / 1024) in LDS
    double top;
    double per, far;                      // 1024 log2(e) / T, and a difference at which the weight is 2^-60
    double least;                         // min_p, in multiples of 2^-shift
    int shift;

    // The weight of a finite logit, in multiples of 2^-shift, with its fraction.  Without branches, so that several are formed
    // side by side; of -inf and of what is no number anything.
    __device__ double scaled(float l) const
    {
        constexpr double round = 1.5 * kMagic, c = 0.69314718055994530942 / kTable;
        const double d = fmax((double)l - top, far);
        const double t = fma(d, per, round), f = fma(d, per, round - t);
        const unsigned n = (unsigned)__builtin_bit_cast(u64, t);           // x as the nearest whole number
        const double e = fma(fma(c * c / 2.0, f, c + c * c * c / 32.0), f, 1.0) * table[n & (kTable - 1)];
        return __builtin_bit_cast(double, __builtin_bit_cast(u64, e) + ((u64)(unsigned)(((int)n >> 10) + shift) << 52));
    }

    static __device__ u64 whole(double scaled) { return __builtin_bit_cast(u64, scaled + kMagic) & 0xFFFFFFFFFFFFFull; }

    __device__ u64 mass(float l) const { return whole(scaled(l)); }

    // with min_p
    __device__ u64 kept(float l) const
    {
        const double w = scaled(l);
        return w >= least ? whole(w) : 0;
    }
};

__device__ inline u64 from_halves(int lo, int hi) { return (u64)(unsigned)hi << 32 | (unsigned)lo; }

// Inclusive prefix sum over the wave, by the lanes' own exchange paths as wave_scan.
__device__ inline u64 wave_scan64(u64 v)
{
#define LORA_SCAN64(CTRL, ROWS)                                                                      \
    v += from_halves(__builtin_amdgcn_update_dpp(0, (int)v, CTRL, ROWS, 0xf, false),                 \
                     __builtin_amdgcn_update_dpp(0, (int)(v >> 32), CTRL, ROWS, 0xf, false));
    LORA_SCAN64(0x111, 0xf)
    LORA_SCAN64(0x112, 0xf)
    LORA_SCAN64(0x114, 0xf)
    LORA_SCAN64(0x118, 0xf)
    LORA_SCAN64(0x142, 0xa)
    LORA_SCAN64(0x143, 0xc)
#undef LORA_SCAN64
    return v;
}

__device__ inline u64 last_lane64(u64 v)
{
    return from_halves(__builtin_amdgcn_readlane((int)v, 63), __builtin_amdgcn_readlane((int)(v >> 32), 63));
}

__device__ inline u64 wave_sum64(u64 v) { return last_lane64(wave_scan64(v)); }

// A border in the order: the tokens above `value`, and the first `ties` of those equal to it.
struct Border {
    float value;
    unsigned ties;
};

template <int THREADS>
struct Shared {
    static constexpr int WAVES = THREADS / 64;
    static constexpr int BINS = 256;                     // of falling logits, over 32 powers of two of weights, for every wave
    static constexpr int COUNTS = 4 * THREADS;           // the same over 48, beyond which no token has a weight
    static constexpr int FINE = THREADS;                 // of the values' bits
    // tokens of a list: as many as LDS holds, for bins with more are read from the row again, three times (64 rows of 200000 273 us with
    // a list of 4096, now 162)
    static constexpr int LISTED = THREADS == 1024 ? 14336 : THREADS == 512 ? 6144 : 1024;
    // tokens of a list that are compared in pairs (400 of 512 tokens 64 us, in bins 28)
    static constexpr int FEW = THREADS > 256 ? 256 : 128;
    double table[kTable];
    union {
        u64 mass[WAVES][BINS];
        unsigned count[COUNTS];
        struct {
            u64 mass[FINE];
            unsigned count[FINE];
        } fine;
        u64 pair_mass[FEW];
    };
    u64 list[LISTED];                     // tokens: keys and, falling, numbers
    u64 wave_mass[WAVES], wave_kept[WAVES];
    unsigned wave_count[WAVES];
    float wave_top[WAVES], wave_low[WAVES];
    int wave_at[WAVES];
    unsigned listed, lo, hi;
    // what a scan has found
    int bin;
    u64 before;
};

// Of the threads' bins, EACH of a thread's own, the first one with which the sum reaches `want`, in sh.bin, and the sum before it in
// sh.before.  -1 and the whole sum if there is none.  Ends with every thread past a barrier.
template <int THREADS, int EACH, class T>
__device__ inline void find_bin(Shared<THREADS> &sh, const T (&own)[EACH], u64 want)
{
    constexpr int WAVES = THREADS / 64;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    u64 m = 0;
#pragma unroll
    for (int k = 0; k < EACH; ++k) m += own[k];
    const u64 upto = wave_scan64(m);
    if (lane == 63) sh.wave_mass[wave] = upto;
    __syncthreads();
    u64 before = upto - m, all = 0;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
        if (w == wave) before += all;
        all += sh.wave_mass[w];
    }
    if (all < want) {
        if (tid == 0) sh.bin = -1, sh.before = all;
    } else if (before < want && before + m >= want) {   // one thread
        int k = 0;
#pragma unroll
        for (; k < EACH - 1; ++k) {
            if (before + own[k] >= want) break;
            before += own[k];
        }
        sh.bin = tid * EACH + k;
        sh.before = before;
    }
    __syncthreads();
}

// A listed token: larger ones come first in the order.
__device__ inline u64 entry_of(unsigned key, int number) { return (u64)key << 32 | (unsigned)~number; }
__device__ inline unsigned key_in(u64 entry) { return (unsigned)(entry >> 32); }
__device__ inline int number_in(u64 entry) { return (int)~(unsigned)entry; }

template <bool F32, int THREADS>
__global__ __launch_bounds__(THREADS, 4) void sample_kernel(SampleParams p)
{
    typedef Shared<THREADS> Lds;
    constexpr int WAVES = THREADS / 64, VEC = Row<F32>::VEC, BINS = Lds::BINS, FINE = Lds::FINE, COUNTS = Lds::COUNTS;
    constexpr int FINE_BITS = 31 - __builtin_clz(FINE);
    __shared__ Lds sh;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int64_t r = blockIdx.x;
    const Row<F32> row(p.logits, r * p.ld, p.vocab);
    // a wave's stretch of the vocabulary is `steps` times 64 lanes' pieces
    const int pieces = row.pieces(), steps = (pieces + THREADS - 1) / THREADS, begin = wave * steps * 64 + lane;
    // every thread: its pieces of `count` steps, AHEAD of them at a time, the next ones on their way meanwhile: more where little
    // is done with them, as all that is done stands there as often
    const std::integral_constant<bool, true> yes;
    const std::integral_constant<bool, false> no;
    const std::integral_constant<int, 1> one;
    const std::integral_constant<int, F32 ? 2 : 1> some;
    const std::integral_constant<int, F32 ? 4 : 2> many;
    const std::integral_constant<int, 8> most;
    const auto each_group = [&](auto ahead, int from, int count, auto f) {
        constexpr int AHEAD = decltype(ahead)::value;
        constexpr bool WAIT = AHEAD == decltype(most)::value;      // as many as there are registers for: none besides
        u32x4 v[AHEAD], next[AHEAD];
        const auto fetch = [&](int k) {
#pragma unroll
            for (int j = 0; j < AHEAD; ++j) next[j] = row.load(k + j < count ? from + (k + j) * 64 : pieces);
        };
        if (!WAIT) fetch(0);
        for (int k = 0; k < count; k += AHEAD) {
            if (WAIT) fetch(k);
#pragma unroll
            for (int j = 0; j < AHEAD; ++j) v[j] = next[j];
            if (!WAIT) fetch(k + AHEAD);
            f(v, from + k * 64);
        }
    };
    const auto each_piece = [&](auto ahead, int from, int count, auto f) {
        each_group(ahead, from, count, [&](auto &v, int i) {
#pragma unroll
            for (int j = 0; j < decltype(ahead)::value; ++j) f(v[j], i + j * 64);
        });
    };
    const auto each = [&](auto ahead, auto f) {
        each_piece(ahead, begin, steps, [&](u32x4 v, int i) {
#pragma unroll
            for (int e = 0; e < VEC; ++e) f(Row<F32>::at(v, e), row.number(i, e));
        });
    };
    const float T = p.temperature ? p.temperature[r] : 1.f;
    const int k_most = p.top_k ? p.top_k[r] : 0;
    const float top_p = p.top_p ? p.top_p[r] : 1.f, min_p = p.min_p ? p.min_p[r] : 0.f, u = p.u[r];
    const bool greedy = !(T > 0.f);
    for (int i = tid; i < kTable; i += THREADS) sh.table[i] = exp2(i / (double)kTable);

    // 1: the largest logit
    float mine = -INFINITY;
    each(most, [&](float l, int) { mine = fmaxf(mine, l); });
    float top = mine, low = mine > -INFINITY ? mine : INFINITY;          // low: the least of the threads' largest
#pragma unroll
    for (int d = 32; d; d >>= 1) top = fmaxf(top, __shfl_xor(top, d)), low = fminf(low, __shfl_xor(low, d));
    if (lane == 0) sh.wave_top[wave] = top, sh.wave_low[wave] = low;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < WAVES; ++w) top = fmaxf(top, sh.wave_top[w]), low = fminf(low, sh.wave_low[w]);
    if (top == -INFINITY || greedy) {
        int at = INT_MAX;                 // the first place that has it
        if (mine == top)
            each(one, [&](float l, int i) {
                if (l == top) at = min(at, i);
            });
#pragma unroll
        for (int d = 32; d; d >>= 1) at = min(at, __shfl_xor(at, d));
        if (lane == 0) sh.wave_at[wave] = at;
        __syncthreads();
        if (tid == 0) {
            for (int w = 1; w < WAVES; ++w) at = min(at, sh.wave_at[w]);
            p.token[r] = top == -INFINITY ? -1 : at;
            if (p.prob) p.prob[r] = top == -INFINITY ? 0.f : 1.f;
        }
        return;
    }

    // with an infinite largest logit only its equals have a weight, and it is the border's value from the start
    const bool endless = top == INFINITY;
    Weigh weigh;
    weigh.table = sh.table;
    weigh.top = top;
    weigh.per = kTable * 1.4426950408889634074 / (double)T;
    weigh.far = -60.0 * kTable / weigh.per;
    weigh.least = min_p > 0.f ? __builtin_ldexp((double)fminf(min_p, 1.f), p.shift) : 0.0;
    weigh.shift = p.shift;
    const Bins by_weight = bins_over(32.f, BINS, T), by_number = bins_over(48.f, COUNTS, T);
    const float at_u = u > 0.f ? fminf(u, 0x1.fffffep-1f) : 0.f;
    const auto goal_of = [&](u64 total) { return min((u64)((double)at_u * (double)total), total - 1); };
    const auto chosen = [&](int i, float l, u64 total) {
        p.token[r] = i;
        if (p.prob) p.prob[r] = (float)((endless ? __builtin_ldexp(1.0, p.shift) : weigh.scaled(l)) / (double)total);
    };
    // top_p of a weight: at least so much is kept
    const auto part_of = [&](u64 all) {
        const double part = ceil((double)top_p * (double)all);
        return part < 1.0 ? 1 : min((u64)part, all);
    };
    // Sum over the workgroup.
    const auto sum_of = [&](u64 x) {
        x = wave_sum64(x);
        __syncthreads();
        if (lane == 0) sh.wave_mass[wave] = x;
        __syncthreads();
        x = 0;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) x += sh.wave_mass[w];
        return x;
    };
    // Lists the tokens for which f holds; their number, which may be more than the list takes, and the range of their keys.  f holds for
    // nothing that is -inf: so only the row's own logits are listed.
    const auto list = [&](auto dense, auto f, unsigned &lo, unsigned &hi) {
        __syncthreads();
        if (tid == 0) sh.listed = 0, sh.lo = 0xFFFFFFFFu, sh.hi = 0;
        __syncthreads();
        unsigned a = 0xFFFFFFFFu, b = 0;
        if (!decltype(dense)::value) {
            each(most, [&](float l, int i) {
                if (!f(l)) return;
                const unsigned key = key_of(l), at = atomicAdd(&sh.listed, 1u);
                a = min(a, key);
                b = max(b, key);
                if (at < Lds::LISTED) sh.list[at] = entry_of(key, i);
            });
        } else {
            // a lane's tokens of several pieces, then one place for all of the wave's; their logits are fetched again once they
            // are listed, as picking them out of registers takes longer
            each_group(many, begin, steps, [&](auto &v, int i) {
                unsigned mine = 0;
#pragma unroll
                for (int j = 0; j < decltype(many)::value; ++j)
#pragma unroll
                    for (int e = 0; e < VEC; ++e) mine |= (f(Row<F32>::at(v[j], e)) ? 1u : 0u) << (j * VEC + e);
                if (!__any(mine)) return;
                const unsigned n = __popc(mine), upto = wave_scan(n), n_all = last_lane(upto);
                unsigned at = 0;
                if (lane == 0) at = atomicAdd(&sh.listed, n_all);
                at = __builtin_amdgcn_readfirstlane(at) + upto - n;
                for (; mine; mine &= mine - 1, ++at) {
                    const int bit = __ffs(mine) - 1;
                    if (at < Lds::LISTED) sh.list[at] = (unsigned)row.number(i + bit / VEC * 64, bit % VEC);
                }
            });
            __syncthreads();
            for (unsigned i = tid; i < min(sh.listed, (unsigned)Lds::LISTED); i += THREADS) {
                const int number = (int)sh.list[i];
                const unsigned key = key_of(row.one(number));
                a = min(a, key);
                b = max(b, key);
                sh.list[i] = entry_of(key, number);
            }
            if (sh.listed > Lds::LISTED) a = key_of(-INFINITY), b = key_of(INFINITY);
        }
        if (a <= b) atomicMin(&sh.lo, a), atomicMax(&sh.hi, b);
        __syncthreads();
        lo = sh.lo;
        hi = sh.hi;
        return sh.listed;
    };
    // The border at which the listed tokens with keys lo .. hi, or if they are too many those of the row for which f holds, number `want` or
    // weigh as much; `above` of it lies above hi.
    const auto refine = [&](auto weighed, auto f, unsigned lo, unsigned hi, unsigned n, u64 want, u64 above) {
        constexpr bool MASS = decltype(weighed)::value;
        while (lo < hi) {
            // bins of falling keys: hi - key in steps of a power of two
            const int by = max(0, 32 - __clz(hi - lo) - FINE_BITS);
            __syncthreads();
            if (MASS) sh.fine.mass[tid] = 0;
            else sh.fine.count[tid] = 0;
            __syncthreads();
            const auto put = [&](unsigned key) {
                if (key < lo || key > hi) return;
                if (MASS) atomicAdd(&sh.fine.mass[(hi - key) >> by], weigh.mass(of_key(key)));
                else atomicAdd(&sh.fine.count[(hi - key) >> by], 1u);
            };
            if (n > Lds::LISTED) {
                each(one, [&](float l, int) {
                    if (f(l)) put(key_of(l));
                });
            } else {
                for (unsigned i = tid; i < n; i += THREADS) put(key_in(sh.list[i]));
            }
            __syncthreads();
            if (MASS) find_bin<THREADS, 1>(sh, {sh.fine.mass[tid]}, want - above);
            else find_bin<THREADS, 1>(sh, {sh.fine.count[tid]}, want - above);
            above += sh.before;
            const unsigned far = hi - ((unsigned)sh.bin << by);
            const unsigned wide = (1u << by) - 1u;
            lo = far - lo > wide ? far - wide : lo;
            hi = far;
        }
        const u64 each_one = MASS ? max(weigh.mass(of_key(hi)), (u64)1) : 1;
        return Border{of_key(hi), (unsigned)((want - above + each_one - 1) / each_one)};
    };
    
    Border border{endless ? INFINITY : -INFINITY, endless ? 0xFFFFFFFFu : 0u};
    const bool by_k = k_most > 0 && k_most < p.vocab && !endless, by_p = top_p < 1.f && !endless;
    unsigned listed = 0, lo = 0, hi = 0;
    bool in_list = false;                 // all tokens down to top_k's border are listed
    // 2: the first k of the order
    if (by_k) {
        const u64 want = (u64)k_most;
        float per = low < top ? (float)FINE / (top - low) : 1.f;
        if (k_most <= THREADS / 4 * 3 && per > 0.f && per < 1e30f) {
            // bins of the threads' largest, from the row's down to the least of them
            sh.fine.count[tid] = 0;
            __syncthreads();
            if (mine > -INFINITY) atomicAdd(&sh.fine.count[(int)fminf((top - mine) * per, (float)(FINE - 1))], 1u);
            __syncthreads();
            find_bin<THREADS, 1>(sh, {sh.fine.count[tid]}, want);
            // tokens of that bin and of those before it: by the same function, so that none of the k is missed.  All, where fewer
            // than k threads have any, if no difference is too large
            if (sh.bin < 0) per = 0x1p-100f;
            const float end = sh.bin < 0 || sh.bin == FINE - 1 ? INFINITY : (float)(sh.bin + 1);
            listed = list(no, [&](float l) { return (top - l) * per < end; }, lo, hi);
            in_list = listed <= Lds::LISTED && (sh.bin >= 0 || top < 0x1p102f);
        }
        if (in_list && listed <= Lds::FEW) {
            // `side` neighbouring threads per token, each for every side-th of the others
            int shift = 0;
            while ((listed << (shift + 1)) <= THREADS && shift < 6) ++shift;
            const unsigned side = 1u << shift, i = tid >> shift;
            const u64 entry = i < listed ? sh.list[i] : 0;
            if (tid < listed) sh.pair_mass[tid] = weigh.mass(of_key(key_in(sh.list[tid])));
            __syncthreads();
            const u64 own = i < listed ? sh.pair_mass[i] : 0;
            unsigned rank = 0;
            u64 before = 0;
            if (i < listed) {
#pragma unroll 4
                for (unsigned j = tid & (side - 1); j < listed; j += side) {
                    const bool first = sh.list[j] > entry;
                    rank += first;
                    before += first ? sh.pair_mass[j] : 0;
                }
            }
            for (unsigned d = 1; d < side; d <<= 1) {
                rank += __shfl_xor((int)rank, d);
                before += from_halves(__shfl_xor((int)before, d), __shfl_xor((int)(before >> 32), d));
            }
            const bool lead = i < listed && (tid & (side - 1)) == 0;
            bool keep = i < listed && rank < (unsigned)k_most;
            if (by_p) keep &= before < part_of(sum_of(lead && keep ? own : 0));
            keep &= weigh.scaled(of_key(key_in(entry))) >= weigh.least;
            const u64 total = sum_of(lead && keep ? own : 0);
            if (lead) sh.pair_mass[i] = keep ? own : 0;
            __syncthreads();
            const u64 goal = goal_of(total);
            before = 0;
            if (i < listed) {
#pragma unroll 4
                for (unsigned j = tid & (side - 1); j < listed; j += side)
                    if (number_in(sh.list[j]) < number_in(entry)) before += sh.pair_mass[j];
            }
            for (unsigned d = 1; d < side; d <<= 1)
                before += from_halves(__shfl_xor((int)before, d), __shfl_xor((int)(before >> 32), d));
            if (lead && keep && before <= goal && goal < before + own) chosen(number_in(entry), of_key(key_in(entry)), total);
            return;
        }
        const auto all = [](float) { return true; };
        if (in_list) {
            if (listed >= want) border = refine(no, all, lo, hi, listed, want, 0);
        } else {
            for (int i = tid; i < COUNTS; i += THREADS) sh.count[i] = 0;
            __syncthreads();
            each(some, [&](float l, int) {
                const int b = bin_of(top, l, by_number);
                if (b < COUNTS) atomicAdd(&sh.count[b], 1u);
            });
            __syncthreads();
            unsigned own[COUNTS / THREADS];
#pragma unroll
            for (int k = 0; k < COUNTS / THREADS; ++k) own[k] = sh.count[tid * (COUNTS / THREADS) + k];
            find_bin(sh, own, want);
        }
        // a border behind the bins cuts nothing that has a weight; but where T is so small that they are of no use all tokens are there
        const bool useless = !(by_number.each < INFINITY);
        if (!in_list && (sh.bin >= 0 || useless)) {
            const int bin = sh.bin < 0 ? COUNTS : sh.bin;
            u64 above = sh.before;
            Bin it = only_bin(by_number, bin);
            // if the list takes the bins above as well, no later step needs the row: 64 rows of 128000 with mixed limits 112.5 -> 98.4 us,
            // 300 of 32000 72.2 -> 57.5 (not if the list is an eighth of the row at most: 72.7); small rows lose, one of 4000 17.1 -> 20.7
            const bool whole = bin < COUNTS && above + sh.count[min(bin, COUNTS - 1)] <= (u64)min(Lds::LISTED, p.vocab / kListedOf) && p.vocab > kSmallVocab;
            if (whole) it.begin = -INFINITY, above = 0;
            const auto in_bin = [=](float l) { return is_in(top, l, -INFINITY, it); };
            listed = list(yes, in_bin, lo, hi);
            in_list = whole && listed <= (unsigned)Lds::LISTED;
            // fewer tokens than that where many are no numbers: all are left
            if (above + listed >= want) border = refine(no, in_bin, lo, hi, listed, want, above);
        }
    }
    // kept weights of this wave's stretch above the border, and the number of those equal to it
    u64 m = 0;
    unsigned c = 0;
    bool summed = false;
    // 3: the border of top_p
    if (in_list) {
        summed = true;                    // nothing that is kept is not listed
        if (by_p) {
            u64 left = 0;
            for (unsigned i = tid; i < listed; i += THREADS) {
                const float l = of_key(key_in(sh.list[i]));
                if (l > border.value) left += weigh.mass(l);
            }
            const u64 above = sum_of(left), tie = weigh.mass(border.value), want = part_of(above + tie * border.ties);
            const auto all = [](float) { return true; };
            if (want > above) border.ties = (unsigned)((want - above + tie - 1) / tie);
            else border = refine(yes, all, key_of(border.value) + 1, hi, listed, want, 0);
        }
    } else if (by_p) {
        u64 tail = 0;                     // weights behind the bins
        __syncthreads();
        for (int i = tid; i < WAVES * BINS; i += THREADS) sh.mass[0][i] = 0;
        __syncthreads();
        const float from = border.value;
        each_piece(some, begin, steps, [&](u32x4 v, int) {
#pragma unroll
            for (int e0 = 0; e0 < VEC; e0 += 4) {
                u64 x[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) x[e] = weigh.mass(Row<F32>::at(v, e0 + e));
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float l = Row<F32>::at(v, e0 + e);
                    const int b = bin_of(top, l, by_weight);
                    if (!(l > from)) continue;
                    if (b < BINS) atomicAdd(&sh.mass[wave][b], x[e]);
                    else tail += x[e];
                }
            }
        });
        __syncthreads();
        u64 own[1] = {0};
        if (tid < BINS)
#pragma unroll
            for (int w = 0; w < WAVES; ++w) own[0] += sh.mass[w][tid];
        const u64 above = sum_of(own[0] + tail);
        // the border's value counts `ties` times
        const u64 tie = from > -INFINITY ? weigh.mass(from) : 0;
        const u64 want = part_of(above + tie * border.ties);
        __syncthreads();
        if (want > above) {               // among top_k's own ties
            border.ties = (unsigned)((want - above + tie - 1) / tie);
        } else {
            find_bin(sh, own, want);
            const int bin = sh.bin < 0 ? BINS : sh.bin;
            const u64 before = sh.before;
            // what each wave's stretch has in the bins above
            u64 mine_above = 0;
            for (int b = lane; b < bin; b += 64) mine_above += sh.mass[wave][b];
            m = wave_sum64(mine_above);
            const Bin it = only_bin(by_weight, bin);
            const auto in_bin = [=](float l) { return is_in(top, l, from, it); };
            listed = list(yes, in_bin, lo, hi);
            border = refine(yes, in_bin, lo, hi, listed, want, before);
            // where min_p is the narrower limit the sums are not those of what is kept
            summed = listed <= Lds::LISTED && weigh.scaled(border.value) >= weigh.least;
        }
    }

    // 4: the token
    const u64 tie_mass = endless ? (u64)1 << p.shift : border.value > -INFINITY ? weigh.kept(border.value) : 0;
    // below this, min_p leaves nothing: ln(min_p) T below the largest, and a little more than what the rounding of either may take, or that of
    // a weight: at min_p = 1 all tokens count whose weights are one in 64 bits
    float least_l = border.value;
    if (min_p > 0.f && !endless) {
        const float far = (1e-6f - logf(fminf(min_p, 1.f))) * T;
        least_l = fmaxf(least_l, top - far * 1.0001f - (fabsf(top) + far) * 1e-6f);
    }
    // kept tokens of a piece above the border, and those equal to it
    const auto look = [&](u32x4 v, u64 &m, unsigned &c) {
        bool any = false;
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
            any |= Row<F32>::at(v, e) >= least_l;
            c += Row<F32>::at(v, e) == border.value;
        }
        if (!__any(any)) return;
#pragma unroll
        for (int e0 = 0; e0 < VEC; e0 += 4) {
            double x[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] = weigh.scaled(Row<F32>::at(v, e0 + e));
#pragma unroll
            for (int e = 0; e < 4; ++e) m += Weigh::whole(Row<F32>::at(v, e0 + e) > border.value && x[e] >= weigh.least ? x[e] : 0.0);
        }
    };
    const auto share = [&](u64 m, unsigned c) {       // a wave's sums, for all to see
        m = wave_sum64(m);
        c = last_lane(wave_scan(c));
        __syncthreads();
        if (lane == 0) sh.wave_kept[wave] = m, sh.wave_count[wave] = c;
        __syncthreads();
    };
    if (summed) {
        share(lane == 0 ? m : 0, 0);
        for (unsigned i = tid; i < listed; i += THREADS) {         // and the border's bin
            const u64 entry = sh.list[i];
            const float l = of_key(key_in(entry));
            const int w = (number_in(entry) + row.skew) / VEC / (steps * 64);
            if (l > border.value) atomicAdd(&sh.wave_kept[w], weigh.kept(l));
            else if (l == border.value) atomicAdd(&sh.wave_count[w], 1u);
        }
        __syncthreads();
    } else {
        m = 0;
        each_piece(some, begin, steps, [&](u32x4 v, int) { look(v, m, c); });
        share(m, c);
    }
    u64 total = 0;
    unsigned all = 0;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) total += sh.wave_kept[w], all += sh.wave_count[w];
    if (endless) {                        // the limits of top_k and top_p among equal weights
        if (k_most > 0) all = min(all, (unsigned)k_most);
        if (top_p < 1.f) all = (unsigned)part_of(all);
        border.ties = all;
    }
    total += min(all, border.ties) * tie_mass;
    u64 goal = goal_of(total);
    unsigned ties = border.ties;
    // The wave in whose part the goal is reached; the goal and the ties that are left at its beginning.
    const auto wave_at = [&] {
        int w = 0;
        for (; w < WAVES - 1; ++w) {
            const unsigned t = min(sh.wave_count[w], ties);
            const u64 weight = sh.wave_kept[w] + t * tie_mass;
            if (goal < weight) break;
            goal -= weight;
            ties -= t;
        }
        return w;
    };
    // the stretch in equal parts for all waves, then the steps of one part
    const int part = (steps + WAVES - 1) / WAVES, from = wave_at() * steps;
    const auto count_of = [&](int w) { return max(0, min(part, steps - w * part)); };
    m = 0;
    c = 0;
    each_piece(one, (from + wave * part) * 64 + lane, count_of(wave), [&](u32x4 v, int) { look(v, m, c); });
    share(m, c);
    const int last = wave_at();
    if (wave != last) return;
    u32x4 hit = {0u, 0u, 0u, 0u};
    int hit_at = -1;
    each_piece(one, (from + last * part) * 64 + lane, count_of(last), [&](u32x4 v, int i) {
        if (hit_at >= 0) return;          // the same for all lanes
        u64 m = 0;
        unsigned c = 0;
        look(v, m, c);
        const unsigned t = min(last_lane(wave_scan(c)), ties);
        const u64 weight = wave_sum64(m) + t * tie_mass;
        if (goal < weight) {
            hit = v;
            hit_at = i - lane;
            return;
        }
        goal -= weight;
        ties -= t;
    });
    m = 0;
    c = 0;
    look(hit, m, c);
    const unsigned before_c = wave_scan(c) - c;
    const u64 own = m + (min(before_c + c, ties) - min(before_c, ties)) * tie_mass, upto = wave_scan64(own);
    if (hit_at < 0 || goal < upto - own || goal >= upto) return;
    u64 sum = upto - own;                 // one lane is left
    unsigned tie = before_c;
#pragma unroll 1
    for (int e = 0; e < VEC; ++e) {
        const float l = Row<F32>::at(hit, 0);
        u64 here = l > border.value ? weigh.kept(l) : 0;
        if (l == border.value && tie++ < ties) here = tie_mass;
        if (sum <= goal && goal < sum + here) chosen(row.number(hit_at + lane, e), l, total);
        sum += here;
        // the next logit comes to the front
        if (F32) hit = u32x4{hit[1], hit[2], hit[3], 0u};
        else hit = u32x4{hit[0] >> 16 | hit[1] << 16, hit[1] >> 16 | hit[2] << 16, hit[2] >> 16 | hit[3] << 16, hit[3] >> 16};
    }
}

template <bool F32>
void launch(const SampleParams &p, hipStream_t s)
{
    if (p.vocab <= (p.n_rows > kRowsAlone ? kTinyVocabMany : kTinyVocab)) hipLaunchKernelGGL((sample_kernel<F32, 256>), dim3(p.n_rows), dim3(256), 0, s, p);
    else if (p.n_rows > kRowsAlone || p.vocab <= kSmallVocab) hipLaunchKernelGGL((sample_kernel<F32, 512>), dim3(p.n_rows), dim3(512), 0, s, p);
    else hipLaunchKernelGGL((sample_kernel<F32, 1024>), dim3(p.n_rows), dim3(1024), 0, s, p);
}

}  // namespace

hipError_t launch_sample(const SampleParams &p, int f32, hipStream_t s)
{
    if (f32) launch<true>(p, s);
    else launch<false>(p, s);
    return hipGetLastError();
}

}  // namespace lora
