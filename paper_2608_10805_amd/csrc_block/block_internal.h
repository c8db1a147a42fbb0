// Kernel arguments and launchers of the operators around the convolution
// (layer norm, scaled residual, AdamW). Internal; not part of the public ABI.
#pragma once

#include <stddef.h>
#include <stdint.h>

#include <hip/hip_runtime_api.h>

#include "wtconv.h"

namespace wtc {

constexpr int64_t kMaxThreads = (int64_t)1 << 32;  // threads of one launch stay below, along each dimension

struct NormArgs {
    const void* x;
    const void* dy;
    const float* w;
    const float* b;
    void* out;           // y or dx
    float* mean;         // written by the forward (or null), read by the backward
    float* rstd;
    float* part;         // backward: nparts rows of 2 C sums (d_weight, then d_bias)
    int64_t B, S, N;     // N = B * S pixels
    int64_t x_stride, dy_stride;
    int C, nparts;
    float eps;
};

struct ResidualArgs {
    const void* x;       // x (forward) or dy (backward), planes
    const void* z;       // rows
    const float* gamma;
    const float* keep;   // one factor an image, or null
    void* out;           // y (planes) or dz (rows, or null)
    float* part;         // backward: nparts rows of C sums, or null
    int64_t B, S, N;
    int C, nparts;
};

// One launch of AdamW: the arguments of its tensors travel with the launch (at
// most 4 KB of kernel arguments), so no table has to be copied or kept.
constexpr int kAdamTensors = 88, kAdamGroups = 8;

struct AdamGroup {
    void *m, *v;
    uint8_t *ms, *vs;
    float b1, omb1, b2, omb2;  // beta1, 1 - beta1, beta2, 1 - beta2
    float rcorr2, eps;         // 1 / sqrt(1 - beta2^t)
    float keep, rate;          // 1 - lr * weight_decay, lr / (1 - beta1^t)
    uint32_t key;
};

struct AdamArgs {
    AdamGroup group[kAdamGroups];
    void* p[kAdamTensors];
    const void* g[kAdamTensors];
    int64_t n[kAdamTensors];
    int64_t at[kAdamTensors];        // first element of its moments
    uint32_t first[kAdamTensors];    // first chunk of each tensor
    uint8_t of[kAdamTensors];        // its group
    uint32_t chunks;                 // of all of them
    int count;
    const float* scale;
};
static_assert(sizeof(AdamArgs) <= 4096, "kernel arguments");

int64_t norm_parts(const wtconv_norm_desc& d);      // rows of partial sums of the backward
int64_t residual_parts(const wtconv_residual_desc& d);

// The kernels that hold every channel of a pixel in registers; false, with
// nothing launched, where there are too many, or more pixels than one launch takes.
bool launch_rows_forward(wtconv_dtype dt, const NormArgs& a, hipStream_t s);
bool launch_rows_backward(wtconv_dtype dt, const NormArgs& a, hipStream_t s);
bool launch_planes_f32(bool forward, bool out_planes, const NormArgs& a, hipStream_t s);
bool launch_planes_bf16(bool forward, bool out_planes, const NormArgs& a, hipStream_t s);
bool launch_planes_f16(bool forward, bool out_planes, const NormArgs& a, hipStream_t s);
int64_t parts_planes_f32(int64_t B, int64_t S, int C);  // workgroups of the backward pass, 0 where it is not theirs
int64_t parts_planes_16(int64_t B, int64_t S, int C);
hipError_t launch_norm_forward(const wtconv_norm_desc& d, const NormArgs& a, hipStream_t s);
hipError_t launch_norm_backward(const wtconv_norm_desc& d, NormArgs a, float* dw, float* db, hipStream_t s);
hipError_t launch_residual_forward(wtconv_dtype dt, const ResidualArgs& a, hipStream_t s);
hipError_t launch_residual_backward(wtconv_dtype dt, ResidualArgs a, float* dgamma, hipStream_t s);
int64_t adam_chunk_elements();
int64_t adam_most_chunks();  // of one launch
hipError_t launch_adamw(wtconv_dtype dt, int bits, const AdamArgs& a, hipStream_t s);
hipError_t launch_adamw_moments(wtconv_dtype dt, int64_t n, const uint8_t* m, const uint8_t* ms, const uint8_t* v,
                                const uint8_t* vs, void* om, void* ov, hipStream_t s);
// out[i] (and, from row width `half` on, out2[i - half]) = sum over rows of part[row][i]
hipError_t launch_sum_parts(const float* part, int64_t rows, int width, int half, float* out, float* out2,
                            hipStream_t s);

}  // namespace wtc
