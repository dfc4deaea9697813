// The next token of a row of logits: a workgroup per row.
//
// All limits cut the order of falling logits (equal ones by number), so what is kept is its beginning: the tokens above a border
// value and the first few, by number, of those that are equal to it.  No sort is needed for that:
//   1  the largest logit
//   2  with top_k or top_p: the weights and numbers of tokens in bins of falling logits; the bin in which the k-th token, or the
//      weight of top_p, is reached; then its tokens in bins of their values' bits, finer each time, until one value is left
//   3  each wave sums the kept weights of its stretch of the vocabulary; the stretch in which u is reached is divided among the
//      waves again, until one wave is left with a few tokens.  How many of the border's value are kept is counted along.
// Without limits 2 falls away, at T = 0 both do.
//
// A weight is 2^x, x = (l - max) log2(e) / T, formed in 64 bits from a table of 2^(j/64) and a polynomial of e^f, |f| <= ln 2 / 128
// (f^5 / 120 is below 2^-44 there), and taken as a whole multiple of 2^-shift: the sums of whole numbers are exact, so threads may
// add them in any order.  It falls with l, as every step of its computation does up to its last bits, and the order itself is that of the logits' bits.
#include <limits.h>

#include <algorithm>

#include "kv_device.h"
#include "step_internal.h"

namespace lora {

namespace {

typedef unsigned long long u64;

constexpr int kBins = 4096;               // of falling logits, over the kOctaves powers of two that a weight may have
constexpr double kOctaves = 48.0;
constexpr int kFine = 1024;               // bins of the values' bits
constexpr int kListed = 2048;             // values of a border bin that are kept in LDS
constexpr double kMagic = 4503599627370496.0;      // 2^52: added to a number below it, leaves its rounding to a whole one in the low bits

// The order of floats as that of whole numbers; -0 and 0 are one value.
__device__ inline unsigned key_of(float l)
{
    const unsigned b = __float_as_uint(l + 0.f);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}

__device__ inline float of_key(unsigned k) { return __uint_as_float(k & 0x80000000u ? k & 0x7FFFFFFFu : ~k); }

template <bool F32>
struct Row {
    const void *base;
    static constexpr int VEC = F32 ? 4 : 8;

    __device__ float one(int i) const
    {
        return F32 ? static_cast<const float *>(base)[i] : __uint_as_float((unsigned)static_cast<const uint16_t *>(base)[i] << 16);
    }

    // VEC logits from i on; rows need not be aligned to more than a logit, which the loads do not ask for
    __device__ void load(int i, float (&x)[VEC]) const
    {
        if (F32) {
            typedef f32x4 __attribute__((aligned(4))) loose;
            const f32x4 v = *(const LORA_GLOBAL loose *)(static_cast<const float *>(base) + i);
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] = v[e];
        } else {
            typedef u32x4 __attribute__((aligned(2))) loose;
            const u32x4 v = *(const LORA_GLOBAL loose *)(static_cast<const uint16_t *>(base) + i);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                x[2 * e] = __uint_as_float(v[e] << 16);
                x[2 * e + 1] = __uint_as_float(v[e] & 0xFFFF0000u);
            }
        }
    }
};

// What a row's weights are formed with.
struct Weigh {
    const double *table;                  // 2^(j / 64) in LDS
    float top;
    double per;                           // log2(e) / T
    double least;                         // min_p
    int shift;

    // x of a logit, the power of two of its weight
    __device__ double power(float l) const
    {
        // with an infinite largest logit only its equals have a weight
        const double d = top == INFINITY ? (l == top ? 0.0 : -INFINITY) : (double)l - (double)top;
        return d * per;
    }

    __device__ double weight(double x) const
    {
        const double t = __builtin_rint(x * 64.0);
        const int n = (int)t;
        const double f = (x * 64.0 - t) * (0.69314718055994530942 / 64.0);
        const double e = fma(fma(fma(fma(f, 1.0 / 24.0, 1.0 / 6.0), f, 0.5), f, 1.0), f, 1.0);
        return __builtin_ldexp(table[n & 63] * e, n >> 6);
    }

    // In multiples of 2^-shift; a logit that is no number, and one too far down, have none.
    __device__ u64 mass(double x) const
    {
        if (!(x > -60.0)) return 0;
        return whole(weight(x));
    }

    __device__ u64 whole(double w) const
    {
        const double scaled = __builtin_ldexp(w, shift) + kMagic;
        return __builtin_bit_cast(u64, scaled) & 0xFFFFFFFFFFFFFull;
    }

    __device__ u64 mass(float l) const { return mass(power(l)); }

    // with min_p
    __device__ u64 kept(float l) const
    {
        const double x = power(l);
        if (!(x > -60.0)) return 0;
        const double w = weight(x);
        return w >= least ? whole(w) : 0;
    }

    __device__ int bin(double x) const { return min(kBins - 1, (int)(-x * (kBins / kOctaves))); }
};

__device__ inline u64 wave_sum(u64 v)
{
#pragma unroll
    for (int d = 32; d; d >>= 1) v += __shfl_xor(v, d);
    return v;
}

__device__ inline u64 wave_scan64(u64 v)
{
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const u64 o = __shfl_up(v, d);
        if (lane >= d) v += o;
    }
    return v;
}

// A border in the order: the tokens above `key`, and the first `ties` of those equal to it.
struct Border {
    unsigned key;
    unsigned ties;
};

template <int THREADS>
struct Shared {
    static constexpr int WAVES = THREADS / 64;
    double table[64];
    u64 mass[kBins];
    unsigned count[kBins];
    u64 fine_mass[kFine];
    unsigned fine_count[kFine];
    unsigned list[kListed];
    u64 wave_mass[WAVES];
    unsigned wave_count[WAVES];
    float wave_top[WAVES];
    int wave_at[WAVES];
    unsigned listed, lo, hi;
    // what a scan has found
    int bin;
    u64 mass_before;
    unsigned count_before;
};

// The first bin with which the tokens number `count`, or weigh `mass`; what stands before it.  False if there is none.
template <int THREADS, int BINS>
__device__ inline bool find_bin(Shared<THREADS> &sh, const u64 *mass, const unsigned *count, bool by_count, u64 want)
{
    constexpr int EACH = BINS / THREADS > 0 ? BINS / THREADS : 1, WAVES = THREADS / 64;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    u64 m = 0;
    unsigned c = 0;
    const bool mine = tid * EACH < BINS;
#pragma unroll
    for (int k = 0; k < EACH; ++k) {
        if (mine) m += mass[tid * EACH + k], c += count[tid * EACH + k];
    }
    const u64 upto_m = wave_scan64(m);
    const unsigned upto_c = wave_scan(c);
    if (lane == 63) sh.wave_mass[wave] = upto_m, sh.wave_count[wave] = upto_c;
    if (tid == 0) sh.bin = -1;
    __syncthreads();
    u64 before_m = upto_m - m;
    unsigned before_c = upto_c - c;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
        if (w < wave) before_m += sh.wave_mass[w], before_c += sh.wave_count[w];
    }
    const u64 had = by_count ? before_c : before_m, has = by_count ? before_c + c : before_m + m;
    if (mine && had < want && has >= want) {           // one thread
        int k = 0;
        for (; k < EACH - 1; ++k) {
            const u64 next = by_count ? before_c + count[tid * EACH + k] : before_m + mass[tid * EACH + k];
            if (next >= want) break;
            before_m += mass[tid * EACH + k];
            before_c += count[tid * EACH + k];
        }
        sh.bin = tid * EACH + k;
        sh.mass_before = before_m;
        sh.count_before = before_c;
    }
    __syncthreads();
    return sh.bin >= 0;
}

template <bool F32, int THREADS>
__global__ __launch_bounds__(THREADS) void sample_kernel(SampleParams p)
{
    constexpr int WAVES = THREADS / 64, VEC = Row<F32>::VEC, STEP = 64 * VEC;
    __shared__ Shared<THREADS> sh;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), V = p.vocab;
    const int64_t r = blockIdx.x;
    const Row<F32> row{F32 ? (const void *)(static_cast<const float *>(p.logits) + r * p.ld)
                           : (const void *)(static_cast<const uint16_t *>(p.logits) + r * p.ld)};
    const float T = p.temperature ? p.temperature[r] : 1.f;
    const bool greedy = !(T > 0.f);

    // every thread: its logits of the vocabulary, whole vectors first
    const auto each = [&](auto f) {
        const int whole = V / VEC * VEC;
        for (int i = tid * VEC; i < whole; i += THREADS * VEC) {
            float x[VEC];
            row.load(i, x);
#pragma unroll
            for (int e = 0; e < VEC; ++e) f(x[e], i + e);
        }
        if (whole + tid < V) f(row.one(whole + tid), whole + tid);
    };

    // 1: the largest, and the first place that has it
    float top = -INFINITY;
    int at = INT_MAX;
    each([&](float l, int i) {
        if (l > top) top = l, at = i;
    });
#pragma unroll
    for (int d = 32; d; d >>= 1) {
        const float o = __shfl_xor(top, d);
        const int oi = __shfl_xor(at, d);
        if (o > top || (o == top && oi < at)) top = o, at = oi;
    }
    if (lane == 0) sh.wave_top[wave] = top, sh.wave_at[wave] = at;
    if (tid < 64) sh.table[tid] = exp2(tid / 64.0);
    __syncthreads();
    top = sh.wave_top[0];
    at = sh.wave_at[0];
#pragma unroll
    for (int w = 1; w < WAVES; ++w)
        if (sh.wave_top[w] > top || (sh.wave_top[w] == top && sh.wave_at[w] < at)) top = sh.wave_top[w], at = sh.wave_at[w];
    if (top == -INFINITY || greedy) {
        if (tid == 0) {
            p.token[r] = top == -INFINITY ? -1 : at;
            if (p.prob) p.prob[r] = top == -INFINITY ? 0.f : 1.f;
        }
        return;
    }

    const int k = p.top_k ? p.top_k[r] : 0;
    const float top_p = p.top_p ? p.top_p[r] : 1.f, min_p = p.min_p ? p.min_p[r] : 0.f;
    const Weigh weigh{sh.table, top, 1.4426950408889634074 / (double)T, min_p > 0.f ? (double)fminf(min_p, 1.f) : 0.0, p.shift};
    Border border{0u, 0u};                // keys are above 0: everything is kept
    const bool by_k = k > 0 && k < V, by_p = top_p < 1.f;

    // 2: the border
    if (by_k || by_p) {
        for (int i = tid; i < kBins; i += THREADS) sh.mass[i] = 0, sh.count[i] = 0;
        __syncthreads();
        each([&](float l, int) {
            const double x = weigh.power(l);
            const u64 m = weigh.mass(x);
            if (m) {
                const int b = weigh.bin(x);
                atomicAdd(&sh.mass[b], m);
                atomicAdd(&sh.count[b], 1u);
            }
        });
        __syncthreads();
        // Where the first bin with `want` tokens, or weight, has it: narrows the bin down to one value.
        const auto refine = [&](bool by_count, u64 want) {
            const int bin = sh.bin;
            u64 mass_before = sh.mass_before;
            unsigned count_before = sh.count_before;
            __syncthreads();
            if (tid == 0) sh.listed = 0, sh.lo = 0xFFFFFFFFu, sh.hi = 0;
            __syncthreads();
            const bool fits = sh.count[bin] <= kListed;
            unsigned lo = 0xFFFFFFFFu, hi = 0;
            each([&](float l, int) {
                const double x = weigh.power(l);
                if (!(x > -60.0) || weigh.bin(x) != bin || !weigh.mass(x)) return;
                const unsigned key = key_of(l);
                lo = min(lo, key);
                hi = max(hi, key);
                if (fits) sh.list[atomicAdd(&sh.listed, 1u)] = key;
            });
            if (lo <= hi) atomicMin(&sh.lo, lo), atomicMax(&sh.hi, hi);
            __syncthreads();
            lo = sh.lo;
            hi = sh.hi;
            const unsigned n = sh.listed;
            while (lo < hi) {
                // bins of falling keys: hi - key in steps of a power of two
                const int bits = 32 - __clz(hi - lo), by = max(0, bits - 10);
                __syncthreads();
                for (int i = tid; i < kFine; i += THREADS) sh.fine_mass[i] = 0, sh.fine_count[i] = 0;
                __syncthreads();
                const auto put = [&](unsigned key) {
                    if (key < lo || key > hi) return;
                    const u64 m = weigh.mass(of_key(key));
                    if (!m) return;
                    atomicAdd(&sh.fine_mass[(hi - key) >> by], m);
                    atomicAdd(&sh.fine_count[(hi - key) >> by], 1u);
                };
                if (fits) {
                    for (unsigned i = tid; i < n; i += THREADS) put(sh.list[i]);
                } else {
                    each([&](float l, int) {
                        const double x = weigh.power(l);
                        if (x > -60.0 && weigh.bin(x) == bin) put(key_of(l));
                    });
                }
                __syncthreads();
                find_bin<THREADS, kFine>(sh, sh.fine_mass, sh.fine_count, by_count, want - (by_count ? count_before : mass_before));
                mass_before += sh.mass_before;
                count_before += sh.count_before;
                const unsigned far = hi - ((unsigned)sh.bin << by);
                lo = max(lo, by ? far - ((1u << by) - 1u) : far);
                hi = far;
            }
            const u64 each_mass = weigh.mass(of_key(hi));
            Border b;
            b.key = hi;
            b.ties = by_count ? (unsigned)want - count_before : (unsigned)((want - mass_before + each_mass - 1) / each_mass);
            __syncthreads();              // the last bin has been read by all
            // the weight up to the border
            if (tid == 0) sh.mass_before = mass_before + b.ties * each_mass;
            __syncthreads();
            return b;
        };
        u64 left = 0;                     // the weight of what top_k leaves
        bool cut = false;
        if (by_k && find_bin<THREADS, kBins>(sh, sh.mass, sh.count, true, (u64)k)) {
            border = refine(true, (u64)k);
            left = sh.mass_before;
            cut = true;
        }
        if (by_p) {
            if (!cut) {
                __syncthreads();
                u64 m = 0;
                for (int i = tid; i < kBins; i += THREADS) m += sh.mass[i];
                m = wave_sum(m);
                if (lane == 0) sh.wave_mass[wave] = m;
                __syncthreads();
#pragma unroll
                for (int w = 0; w < WAVES; ++w) left += sh.wave_mass[w];
            }
            __syncthreads();
            const double goal = ceil((double)top_p * (double)left);
            const u64 want = goal < 1.0 ? 1 : min((u64)goal, left);
            find_bin<THREADS, kBins>(sh, sh.mass, sh.count, false, want);
            border = refine(false, want);
        }
        __syncthreads();
    }

    // 3: the token.  A stretch of the vocabulary, what of u's weight and of the border's ties is left to find in it
    const u64 tie_mass = border.key ? weigh.kept(of_key(border.key)) : 0;
    int lo = 0, hi = V;
    u64 goal = 0, total = 0;
    unsigned ties = border.ties;
    bool first = true;
    const auto look = [&](float l, u64 &m, unsigned &c) {
        const unsigned key = key_of(l);
        if (l == l && key >= border.key) {
            if (key == border.key && border.key) c += 1;
            else m += weigh.kept(l);
        }
    };
    while (first || hi - lo > STEP) {
        const int part = max(STEP, ((hi - lo + WAVES - 1) / WAVES + STEP - 1) / STEP * STEP);
        const int a = min(hi, lo + wave * part), b = min(hi, a + part);
        u64 m = 0;
        unsigned c = 0;
        for (int i = a + lane * VEC; i < b; i += STEP) {
            if (i + VEC <= b) {
                float x[VEC];
                row.load(i, x);
#pragma unroll
                for (int e = 0; e < VEC; ++e) look(x[e], m, c);
            } else {
                for (int j = i; j < b; ++j) look(row.one(j), m, c);
            }
        }
        m = wave_sum(m);
        c = last_lane(wave_scan(c));
        __syncthreads();
        if (lane == 0) sh.wave_mass[wave] = m, sh.wave_count[wave] = c;
        __syncthreads();
        if (first) {
            unsigned all = 0;
            for (int w = 0; w < WAVES; ++w) total += sh.wave_mass[w], all += sh.wave_count[w];
            total += min(all, ties) * tie_mass;
            const float u = p.u[r];
            const double want = u > 0.f ? (double)fminf(u, 0x1.fffffep-1f) * (double)total : 0.0;
            goal = min((u64)want, total - 1);
            first = false;
        }
        int w = 0;
        for (; w < WAVES - 1; ++w) {
            const unsigned t = min(sh.wave_count[w], ties);
            const u64 here = sh.wave_mass[w] + t * tie_mass;
            if (goal < here) break;
            goal -= here;
            ties -= t;
        }
        lo = min(hi, lo + w * part);
        hi = min(hi, lo + part);
    }
    if (wave) return;
    // VEC logits a lane
    float x[VEC];
    u64 m = 0;
    unsigned c = 0;
    const int i = lo + lane * VEC;
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
        x[e] = i + e < hi ? row.one(i + e) : -INFINITY;
        if (i + e < hi) look(x[e], m, c);
    }
    const unsigned before_c = wave_scan(c) - c;
    const unsigned had = min(before_c, ties), has = min(before_c + c, ties);
    const u64 own = m + (has - had) * tie_mass, upto = wave_scan64(own);
    if (goal >= upto - own && goal < upto) {           // one lane
        u64 sum = upto - own;
        unsigned tie = before_c;
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
            u64 m1 = 0;
            unsigned c1 = 0;
            if (i + e < hi) look(x[e], m1, c1);
            if (c1 && tie < ties) m1 = tie_mass;
            tie += c1;
            if (sum <= goal && goal < sum + m1) {
                p.token[r] = i + e;
                if (p.prob) p.prob[r] = (float)(__builtin_ldexp(weigh.weight(weigh.power(x[e])), p.shift) / (double)total);
            }
            sum += m1;
        }
    }
}

template <bool F32>
void launch(const SampleParams &p, hipStream_t s)
{
    if (p.vocab <= 8192) hipLaunchKernelGGL((sample_kernel<F32, 256>), dim3(p.n_rows), dim3(256), 0, s, p);
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
