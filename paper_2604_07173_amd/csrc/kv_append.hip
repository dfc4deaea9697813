// Rotary positions and the append to the paged cache in one pass: q is rotated into q_out, k into its page,
// v goes to its page.  Element pairs of the first `rot` elements of a head turn by t = position * freq:
//   (a, b) -> amplitude * (a cos t - b sin t, a sin t + b cos t).
// The angle is formed in turns in 64 bits and its whole turns are dropped before it is rounded to 32, so that
// long positions lose nothing; products and sums are fp32, rounded to bf16 once.
//
// Every element is read once and written once, so the kernel is bound by memory (by the latency of finding a
// row's sequence and page for small batches).  A workgroup takes one row: its waves find the place of the row
// and the cosines, which all heads share, and pass them on through LDS.  16384 rows of 32 + 8 + 8 heads of 128 take 77 us,
// 5.2 TB/s, more than a plain copy of as much (4.85); 64 rows 4.1 us.
#include "kv_device.h"

namespace lora {

namespace {

constexpr int kMaxPairs = LORA_KV_MAX_HEAD_DIM / 2;
constexpr double kTurn = 0.15915494309189533577;      // 1 / (2 pi)

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

template <bool F32>
__device__ inline float load1(const void *base, int64_t at)
{
    return F32 ? static_cast<const float *>(base)[at]
               : __uint_as_float((unsigned)static_cast<const uint16_t *>(base)[at] << 16);
}

__device__ inline uint16_t to_bf16(float x) { return (uint16_t)pack_bf16_rne(x, x); }

// How a thread's unit of a head is rotated.  kScalar: rotated widths that do not split into units of eight.
enum Units { kHalf, kInterleaved, kScalar };

template <bool F32, Units U>
__global__ __launch_bounds__(256) void append_kernel(AppendParams p)
{
    __shared__ float s_cos[kMaxPairs], s_sin[kMaxPairs];
    __shared__ int64_t s_at;                          // offset of the row's place in the cache, -1 = none
    const int t = blockIdx.x;
    const int tid = threadIdx.x;
    const int half = p.rot >> 1;

    // every wave finds the row's sequence for itself: one load for up to 64 sequences
    int pos = 0;
    if (p.kv_heads || !p.b.position) {
        const int s = wave_find(p.b.row_start, p.b.n_seqs, t);
        const int start = p.b.row_start[s], end = p.b.row_start[s + 1];
        pos = p.b.seq_len[s] - end + t;
        if (p.kv_heads && tid == 0) {
            int64_t at = -1;
            // a row of no sequence would stand where tokens of this one are, or where another one's may be
            if (t < start || t >= end || pos < 0 || pos >= p.b.tokens_max) {
                atomicOr(p.b.status, LORA_STATUS_BAD_LENGTH);
            } else {
                const int page = p.b.table[(int64_t)s * p.b.max_pages + (pos >> p.c.page_shift)];
                if ((unsigned)page < (unsigned)p.c.n_pages)
                    at = page * p.c.page_stride + (int64_t)(pos & ((1 << p.c.page_shift) - 1)) * p.c.token_stride;
                else
                    atomicOr(p.b.status, LORA_STATUS_BAD_PAGE);
            }
            s_at = at;
        }
    }
    if (p.b.position) pos = p.b.position[t];
    for (int i = tid; i < half; i += 256) {
        const double turns = (double)pos * (p.freq[i] * kTurn);
        const float r = (float)(turns - rint(turns));
        float sn, cs;
        sincospif(2.f * r, &sn, &cs);
        s_cos[i] = cs * p.amplitude;
        s_sin[i] = sn * p.amplitude;
    }
    __syncthreads();
    const int64_t at = p.kv_heads ? s_at : -1;

    const int D = p.c.dim;
    const int rot_units = U == kHalf ? p.rot >> 4 : U == kInterleaved ? p.rot >> 3 : half;
    const int units = rot_units + (U == kScalar ? D - p.rot : (D - p.rot) >> 3);
    const int turned = (p.heads + p.kv_heads) * units;
    for (int i = tid; i < turned; i += 256) {
        const int h = i / units, u = i - h * units;
        const bool is_q = h < p.heads;
        if (!is_q && at < 0) continue;
        const void *src = is_q ? p.q : p.k;
        const int64_t from = is_q ? t * p.ldq + (int64_t)h * D : t * p.ldk + (int64_t)(h - p.heads) * D;
        uint16_t *dst = is_q ? p.q_out + t * p.ldqo + (int64_t)h * D : p.c.k + at + (h - p.heads) * p.c.head_stride;
        if (U == kScalar) {
            if (u < half) {
                const int ea = p.pairing == LORA_ROPE_HALF ? u : 2 * u, eb = p.pairing == LORA_ROPE_HALF ? u + half : 2 * u + 1;
                const float a = load1<F32>(src, from + ea), b = load1<F32>(src, from + eb);
                dst[ea] = to_bf16(a * s_cos[u] - b * s_sin[u]);
                dst[eb] = to_bf16(a * s_sin[u] + b * s_cos[u]);
            } else {
                const int e = p.rot + u - half;
                dst[e] = to_bf16(load1<F32>(src, from + e));
            }
        } else if (u >= rot_units) {
            const int e = p.rot + 8 * (u - rot_units);
            float x[8];
            load8<F32>(src, from + e, x);
            store8(dst + e, x);
        } else if (U == kHalf) {
            float a[8], b[8], oa[8], ob[8];
            load8<F32>(src, from + 8 * u, a);
            load8<F32>(src, from + half + 8 * u, b);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float c = s_cos[8 * u + j], s = s_sin[8 * u + j];
                oa[j] = a[j] * c - b[j] * s;
                ob[j] = a[j] * s + b[j] * c;
            }
            store8(dst + 8 * u, oa);
            store8(dst + half + 8 * u, ob);
        } else {
            float x[8], o[8];
            load8<F32>(src, from + 8 * u, x);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float c = s_cos[4 * u + j], s = s_sin[4 * u + j];
                o[2 * j] = x[2 * j] * c - x[2 * j + 1] * s;
                o[2 * j + 1] = x[2 * j] * s + x[2 * j + 1] * c;
            }
            store8(dst + 8 * u, o);
        }
    }
    if (at < 0) return;
    const int vecs = D >> 3;
    for (int i = tid; i < p.kv_heads * vecs; i += 256) {
        const int h = i / vecs, e = 8 * (i - h * vecs);
        float x[8];
        load8<F32>(p.v, t * p.ldv + (int64_t)h * D + e, x);
        store8(p.c.v + at + h * p.c.head_stride + e, x);
    }
}

}  // namespace

hipError_t launch_append(const AppendParams &p, hipStream_t s)
{
    const Units u = p.pairing == LORA_ROPE_HALF ? (p.rot % 16 == 0 ? kHalf : kScalar)
                                                : (p.rot % 8 == 0 ? kInterleaved : kScalar);
    const dim3 grid(p.b.n_rows), block(256);
#define LORA_APPEND(F32)                                                                           \
    switch (u) {                                                                                   \
    case kHalf: hipLaunchKernelGGL((append_kernel<F32, kHalf>), grid, block, 0, s, p); break;      \
    case kInterleaved: hipLaunchKernelGGL((append_kernel<F32, kInterleaved>), grid, block, 0, s, p); break; \
    default: hipLaunchKernelGGL((append_kernel<F32, kScalar>), grid, block, 0, s, p);              \
    }
    if (p.f32) {
        LORA_APPEND(true)
    } else {
        LORA_APPEND(false)
    }
#undef LORA_APPEND
    return hipGetLastError();
}

}  // namespace lora
