// The residual's addition and the norm behind it in one pass: s = x + add, y = s r (w + shift) with r = 1 / sqrt(mean s^2 + eps), in
// fp32.  A row stays in registers between its sum of squares and its outputs (above 32768 columns partly in scratch memory: 64 of a thread's
// 128 registers hold it), so every element is read once and written once
// and the kernel is bound by memory (by latency for a decode batch's few rows): 16384 rows of 4096 columns, bf16, with the residual's sum, the
// bf16 rows and e4m3 ones with a scale for every 128 columns (606 MB) 117 us, 5.2 TB/s, more than a plain copy of as much (4.85);
// 1333 rows of 2056 fp32 columns (41 MB) 11 us; 64 rows 4.5 us, of which a launch takes 3.  Wide rows, 2048 of them in bf16 with e4m3: 16384 columns
// 67 us, 4.5 TB/s; 32768 135 us, 4.5; 65536 392 us, 3.1.
//
// Vector v of a row, eight columns, belongs to thread v % T of the row's T threads: loads are contiguous over a wave, and a group of
// columns that share a scale (8 .. 512) lies in neighbouring lanes of one wave.
#include <algorithm>

#include "lora_device.h"
#include "step_internal.h"

namespace lora {

namespace {

constexpr float kMost8 = 448.f;           // largest e4m3 value
constexpr float kShrink = 0x1p-80f;       // rows whose mean of squares and eps are infinite: 65536 (2^128 2^-80)^2 is far below 2^128

template <bool F32>
__device__ inline void load8(const void *base, int64_t at, float (&x)[8])
{
    if (F32) {
        const float *p = static_cast<const float *>(base) + at;
        const f32x4 a = ld16f(p), b = ld16f(p + 4);
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = a[i], x[4 + i] = b[i];
    } else {
        const u32x4 a = ld16<false>(static_cast<const uint16_t *>(base) + at);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[2 * i] = __uint_as_float(a[i] << 16);
            x[2 * i + 1] = __uint_as_float(a[i] & 0xFFFF0000u);
        }
    }
}

__device__ inline void store8(uint16_t *p, const float (&x)[8])
{
    u32x4 o;
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] = pack_bf16_rne(x[2 * i], x[2 * i + 1]);
    st16<false>(p, o);
}

// Over the threads of a row: LANES neighbouring lanes of a wave, or, 0, all waves of the workgroup through LDS.
template <int LANES, class V, class Op>
__device__ inline V over_row(V v, V *s_part, Op op)
{
#pragma unroll
    for (int d = (LANES ? LANES : 64) / 2; d; d >>= 1) v = op(v, __shfl_xor(v, d));
    if (LANES) return v;
    __syncthreads();                      // a former call's parts have been read
    if ((threadIdx.x & 63) == 0) s_part[threadIdx.x >> 6] = v;
    __syncthreads();
    v = s_part[0];
    for (unsigned w = 1; w < blockDim.x >> 6; ++w) v = op(v, s_part[w]);
    return v;
}

enum Add { kNone, kBf16, kF32 };

// N vectors of a row per thread.  LANES: a row is that many lanes', and a workgroup takes 256 / LANES at a time; 0: all of it takes one.
template <bool XF32, Add A, int LANES, int N>
__global__ __launch_bounds__(LANES ? 256 : 1024) void norm_kernel(NormParams p)
{
    constexpr int SHARE = LANES ? LANES : 256, ROWS = 256 / SHARE;
    __shared__ float s_part[16];
    __shared__ unsigned s_top[16];
    const int T = LANES ? LANES : blockDim.x, t = LANES ? threadIdx.x % SHARE : threadIdx.x;
    for (int64_t row = (int64_t)blockIdx.x * ROWS + (LANES ? threadIdx.x / SHARE : 0); row < p.n_rows; row += (int64_t)gridDim.x * ROWS) {
        float s[N][8];
        float sum = 0.f;
#pragma unroll
        for (int k = 0; k < N; ++k) {
            const int c = (k * T + t) * 8;
            if (c < p.width) {
                load8<XF32>(p.x, row * p.ldx + c, s[k]);
                if (A != kNone) {
                    float a[8];
                    load8<A == kF32>(p.add, row * p.ldadd + c, a);
#pragma unroll
                    for (int i = 0; i < 8; ++i) s[k][i] += a[i];
                }
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) s[k][i] = 0.f;
            }
        }
#pragma unroll
        for (int k = 0; k < N; ++k)
#pragma unroll
            for (int i = 0; i < 8; ++i) sum += s[k][i] * s[k][i];
        const auto plus = [](float a, float b) { return a + b; };
        sum = over_row<LANES>(sum, s_part, plus);
        if (p.sum) {
#pragma unroll
            for (int k = 0; k < N; ++k) {
                const int c = (k * T + t) * 8;
                if (c >= p.width) continue;
                if (XF32) {
                    float *to = static_cast<float *>(p.sum) + row * p.ldsum + c;
                    st16f(to, f32x4{s[k][0], s[k][1], s[k][2], s[k][3]});
                    st16f(to + 4, f32x4{s[k][4], s[k][5], s[k][6], s[k][7]});
                } else {
                    store8(static_cast<uint16_t *>(p.sum) + row * p.ldsum + c, s[k]);
                }
            }
        }
        if (!p.out && !p.out8) continue;
        float mean = sum / (float)p.width + p.eps;
        if (mean == INFINITY) {           // the same for all threads of the row
            sum = 0.f;
#pragma unroll
            for (int k = 0; k < N; ++k)
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    s[k][i] *= kShrink;
                    sum += s[k][i] * s[k][i];
                }
            sum = over_row<LANES>(sum, s_part, plus);
            mean = sum / (float)p.width + p.eps * kShrink * kShrink;
        }
        const float r = 1.f / sqrtf(mean);
        unsigned top = 0;                 // of |y| as bits: a NaN is above all numbers
#pragma unroll
        for (int k = 0; k < N; ++k) {
            const int c = (k * T + t) * 8;
            // (fetched before the row is summed they take registers from other workgroups: 16384 rows of 4096 columns 117 -> 121 us)
            float w[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) w[i] = 1.f;
            if (c < p.width && p.weight) {
                if (p.weight_f32) load8<true>(p.weight, c, w);
                else load8<false>(p.weight, c, w);
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) s[k][i] = s[k][i] * r * (w[i] + p.shift);
            if (c < p.width && p.out) store8(p.out + row * p.ldo + c, s[k]);
        }
        if (!p.out8) continue;
        unsigned tops[N];
#pragma unroll
        for (int k = 0; k < N; ++k) {
            tops[k] = 0;
            if ((k * T + t) * 8 < p.width) {
#pragma unroll
                for (int i = 0; i < 8; ++i) tops[k] = max(tops[k], __float_as_uint(s[k][i]) & 0x7FFFFFFFu);
            }
            top = max(top, tops[k]);
        }
        if (p.group) {
#pragma unroll
            for (int k = 0; k < N; ++k)
                for (int d = 1; d < min(p.group >> 3, LANES ? LANES : 64); d <<= 1) tops[k] = max(tops[k], (unsigned)__shfl_xor((int)tops[k], d));
        } else {
            top = over_row<LANES>(top, s_top, [](unsigned a, unsigned b) { return max(a, b); });
#pragma unroll
            for (int k = 0; k < N; ++k) tops[k] = top;
        }
#pragma unroll
        for (int k = 0; k < N; ++k) {
            const int v = k * T + t, c = v * 8;
            if (c >= p.width) continue;
            const float most = __uint_as_float(tops[k]);
            const float scale = most == 0.f ? 1.f : most / kMost8;
            // y / scale as a product with 1 / scale, and what that leaves of y divided once more: the quotient, rounded once.  Of the smallest
            // values 2^100 times as much, so that nothing is lost below 2^-126; where the largest is infinite, the first product stands
            const float up = most < 1e-20f ? 0x1p100f : 1.f;
            const float by = most * up / kMost8, inv = most == 0.f ? 1.f : 1.f / by, rest_by = most < INFINITY ? by : 0.f;
            const auto over = [=](float y) {
                const float a = y * up, q = a * inv;
                return fmaf(fmaf(-q, rest_by, a), inv, q);
            };
            int packed[2] = {0, 0};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float a = over(s[k][2 * i]), b = over(s[k][2 * i + 1]);
                // what rounding has taken beyond the largest value comes back; a NaN stays one
                const float x = a > kMost8 ? kMost8 : a < -kMost8 ? -kMost8 : a, y = b > kMost8 ? kMost8 : b < -kMost8 ? -kMost8 : b;
                if (i & 1) packed[i >> 1] = __builtin_amdgcn_cvt_pk_fp8_f32(x, y, packed[i >> 1], true);
                else packed[i >> 1] = __builtin_amdgcn_cvt_pk_fp8_f32(x, y, packed[i >> 1], false);
            }
            *reinterpret_cast<u32x2 *>(p.out8 + row * p.ld8 + c) = u32x2{(unsigned)packed[0], (unsigned)packed[1]};
            if (p.group ? (c & (p.group - 1)) == 0 : v == 0) p.scale[row * p.ld_scale + (p.group ? c / p.group : 0)] = scale;
        }
    }
}

template <bool XF32, Add A>
void launch_width(const NormParams &p, hipStream_t s)
{
    const int vecs = p.width / 8;
    // As many lanes or waves as the row fills, so that few have nothing to do (20000 rows of 64 columns in bf16 and e4m3 4.8 to 5.6 us, a wave
    // for each 11.9; of 128 6.7 and 12.4, of 256 10.5 and 13.4).  One vector a thread up to five waves (1333 rows of 2056 fp32 columns
    // 11.0 us, with two 11.4); with eight 16384 rows of 4096 columns gain 2 % and 2130 of 3912 lose 12
#define LORA_NORM(LANES, N)                                                                                    \
    {                                                                                                          \
        const int rows = 256 / (LANES ? LANES : 256), threads = LANES ? 256 : (vecs + 64 * N - 1) / (64 * N) * 64; \
        const int grid = std::min((p.n_rows + rows - 1) / rows, 65536);                                        \
        hipLaunchKernelGGL((norm_kernel<XF32, A, LANES, N>), dim3(grid), dim3(threads), 0, s, p);              \
    }
    if (vecs <= 8) LORA_NORM(8, 1)
    else if (vecs <= 16) LORA_NORM(16, 1)
    else if (vecs <= 32) LORA_NORM(32, 1)
    else if (vecs <= 64) LORA_NORM(64, 1)
    else if (vecs <= 128) LORA_NORM(64, 2)
    else if (vecs <= 320) LORA_NORM(0, 1)
    else if (vecs <= 1024) LORA_NORM(0, 2)
    else if (vecs <= 4096) LORA_NORM(0, 4)
    else LORA_NORM(0, 8)
#undef LORA_NORM
}

}  // namespace

hipError_t launch_norm(const NormParams &p, int x_f32, int add_f32, hipStream_t s)
{
    const Add a = !p.add ? kNone : add_f32 ? kF32 : kBf16;
    if (x_f32) {
        if (a == kNone) launch_width<true, kNone>(p, s);
        else if (a == kBf16) launch_width<true, kBf16>(p, s);
        else launch_width<true, kF32>(p, s);
    } else {
        if (a == kNone) launch_width<false, kNone>(p, s);
        else if (a == kBf16) launch_width<false, kBf16>(p, s);
        else launch_width<false, kF32>(p, s);
    }
    return hipGetLastError();
}

}  // namespace lora
