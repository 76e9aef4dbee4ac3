// Layer norm: the types' kernels, the gradient's workspace and the end of its columns' sums.
#include "aqsgd_layernorm.h"

namespace aqsgd {

#define AQSGD_EXTERN_LAYERNORM(DT)                                                        \
    extern template hipError_t launch_layernorm_as<DT>(const LayernormArgs&, hipStream_t); \
    extern template hipError_t launch_layernorm_grad_as<DT>(const LayernormGradArgs&, hipStream_t);
AQSGD_EXTERN_LAYERNORM(AQSGD_F32)
AQSGD_EXTERN_LAYERNORM(AQSGD_F16)
AQSGD_EXTERN_LAYERNORM(AQSGD_BF16)

int64_t layernorm_grad_workspace_bytes(int dtype, int64_t rows, int64_t cols) {
    const GradPlan p = dtype == AQSGD_F32 ? grad_plan<AQSGD_F32>(rows, cols) : grad_plan<AQSGD_F16>(rows, cols);
    return 2 * p.blocks * cols * 4;
}

// Joins the blocks' sums of 64 columns: four lanes to a column, each every fourth block.  blockIdx.y: weight, bias.
static __global__ __launch_bounds__(256) void layernorm_join_kernel(const LayernormGradArgs a, const int64_t blocks) {
    __shared__ double part[4][64];
    float* out = blockIdx.y == 0 ? a.dweight : a.dbias;
    if (!out) return;
    const float* from = a.workspace + blockIdx.y * blocks * a.cols;
    const int lane = threadIdx.x & 63, slot = threadIdx.x >> 6;
    const int64_t c = static_cast<int64_t>(blockIdx.x) * 64 + lane;
    double s = 0.0;
    if (c < a.cols)
        for (int64_t b = slot; b < blocks; b += 4) s += static_cast<double>(from[b * a.cols + c]);
    part[slot][lane] = s;
    __syncthreads();
    if (slot != 0 || c >= a.cols) return;
    const float sum = static_cast<float>(part[0][lane] + part[1][lane] + part[2][lane] + part[3][lane]);
    out[c] = a.accumulate ? out[c] + sum : sum;
}

hipError_t launch_layernorm_join(const LayernormGradArgs& a, int64_t blocks, hipStream_t stream) {
    return launch_kernel(layernorm_join_kernel, dim3(static_cast<unsigned>((a.cols + 63) / 64), 2), dim3(256), stream, a, blocks);
}

hipError_t launch_layernorm(int dtype, const LayernormArgs& a, hipStream_t stream) {
    switch (dtype) {
    case AQSGD_F32:  return launch_layernorm_as<AQSGD_F32>(a, stream);
    case AQSGD_F16:  return launch_layernorm_as<AQSGD_F16>(a, stream);
    default:         return launch_layernorm_as<AQSGD_BF16>(a, stream);
    }
}

hipError_t launch_layernorm_grad(int dtype, const LayernormGradArgs& a, hipStream_t stream) {
    switch (dtype) {
    case AQSGD_F32:  return launch_layernorm_grad_as<AQSGD_F32>(a, stream);
    case AQSGD_F16:  return launch_layernorm_grad_as<AQSGD_F16>(a, stream);
    default:         return launch_layernorm_grad_as<AQSGD_BF16>(a, stream);
    }
}

}  // namespace aqsgd
