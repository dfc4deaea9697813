// Internal declarations of the residual norm and of sampling (host side; kernels live in norm.hip and sample.hip).
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "../../include/lora_step.h"
#include "lora_layout.h"

namespace lora {

int note_hip_error(hipError_t e);   // keeps the text for lora_last_hip_error; returns LORA_ERR_HIP

struct NormParams {
    const void *x, *add, *weight;
    void *sum;
    uint16_t *out;
    uint8_t *out8;
    float *scale;
    int64_t ldx, ldadd, ldsum, ldo, ld8, ld_scale;
    int n_rows, width, weight_f32, group;     // group: columns of a scale, 0 = the row
    float eps, shift;
};

struct SampleParams {
    const void *logits;
    const float *temperature, *top_p, *min_p, *u;
    const int32_t *top_k;
    int32_t *token;
    float *prob;
    int64_t ld;
    int n_rows, vocab;
    int shift;                                // a weight of one is 2^shift
};

hipError_t launch_norm(const NormParams &p, int x_f32, int add_f32, hipStream_t s);
hipError_t launch_sample(const SampleParams &p, int f32, hipStream_t s);

}  // namespace lora
