// What the layer norm's and the weights' update's entries (aqsgd_layernorm*, aqsgd_adamw, aqsgd_grad_norm) share with
// their kernels: the arguments.
#pragma once

#include "aqsgd_kernels.h"

namespace aqsgd {

// ---- layer norm --------------------------------------------------------------------------------
struct LayernormArgs {
    const void* x;
    const void* residual;
    const void* weight;
    const void* bias;
    void* sum;
    void* y;
    float* mean;
    float* rstd;
    int8_t* codes;
    float* scales;
    int64_t rows, ld;
    int64_t code_stride;                 // bytes
    double eps, each;                    // each: 1 / cols
    int32_t cols;
};
hipError_t launch_layernorm(int dtype, const LayernormArgs& a, hipStream_t stream);

struct LayernormGradArgs {
    const void* dy;
    const void* x;
    const float* mean;
    const float* rstd;
    const void* weight;
    const void* add;
    void* dx;
    float* dweight;
    float* dbias;
    float* workspace;
    int64_t rows, ld;
    int32_t cols;
    int32_t accumulate;
};
int64_t layernorm_grad_workspace_bytes(int dtype, int64_t rows, int64_t cols);
hipError_t launch_layernorm_grad(int dtype, const LayernormGradArgs& a, hipStream_t stream);

// ---- the weights' update -----------------------------------------------------------------------
constexpr int kStateGroup = 256;                 // states that share a scale
constexpr int kTableTensors = 64;                // tensors of a launch: a wave finds a workgroup's with one load and one vote

struct UpdateTensor {
    void* param;
    const void* grad;
    char* state;
    float* master;
    int64_t n;
    int64_t group0;                              // groups of the call's tensors in front of it
    double weight_decay;
    float decay;                                 // 1 - lr * weight_decay
};

// A launch's tensors; first[i]: the first workgroup of tensor i, after the last one a number no workgroup has.
struct UpdateTable {
    uint32_t first[kTableTensors];
    UpdateTensor tensor[kTableTensors];
};

struct AdamwArgs {
    double lr, beta1, beta2;
    int64_t step;
    const float* lr_at;                          // device values that take the places of lr and step, or null
    const int64_t* step_at;
    const float* scale;
    float beta1f, rest1, beta2f, rest2, eps;     // rest: 1 - beta
    float length, correct;                       // lr / (1 - beta1^t), 1 / sqrt(1 - beta2^t)
    uint64_t seed, key;                          // key: seed + t
};
struct AdamwKind {
    int dtype, grad_dtype, state_bits, rounding;
};
// The factors of a step, formed in binary64 by the host and, where lr or the step are on the device, by the kernels: the same
// operations, the same bits.
__host__ __device__ inline double power_of(double base, int64_t n) {
    double p = 1.0;
    for (; n > 0; n >>= 1) {
        if (n & 1) p *= base;
        base *= base;
    }
    return p;
}
__host__ __device__ inline float decay_factor(double lr, double weight_decay) { return static_cast<float>(1.0 - lr * weight_decay); }
__host__ __device__ inline float length_factor(double lr, double beta1, int64_t step) { return static_cast<float>(lr / (1.0 - power_of(beta1, step))); }
__host__ __device__ inline float correct_factor(double beta2, int64_t step) { return static_cast<float>(1.0 / sqrt(1.0 - power_of(beta2, step))); }
int64_t adamw_workgroups(int64_t n);             // of a tensor
hipError_t launch_adamw(const AdamwKind& kind, const UpdateTable& table, uint32_t blocks, const AdamwArgs& a, hipStream_t stream);

// A launch of the norm's first pass: workgroup b leaves the sum of its part's squares in partial[b].
struct NormTable {
    uint32_t first[kTableTensors];
    const void* grad[kTableTensors];
    int64_t n[kTableTensors];
};
hipError_t launch_grad_squares(int dtype, const NormTable& table, uint32_t blocks, int64_t span, double* partial, hipStream_t stream);
// Up to so many chunks of norm_chunk() elements, a tensor's last one shorter, in one launch: first[i] counts chunks.
constexpr int kFewChunks = 64;
int64_t norm_chunk(int dtype);
hipError_t launch_grad_norm_few(int dtype, const NormTable& table, uint32_t chunks, double max_norm, const float* loss_scale, float* result, hipStream_t stream);
hipError_t launch_grad_norm(const double* partial, int64_t count, double max_norm, const float* loss_scale, float* result, hipStream_t stream);

}  // namespace aqsgd
