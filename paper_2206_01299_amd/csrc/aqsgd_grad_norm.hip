// The 2-norm over many tensors' gradients and the factor that clips them: a pass that leaves a sum of squares for each
// workgroup, and one workgroup that joins them.  Squares are summed in binary64, in which none overflows and no order
// shows.  Memory bounds the first pass.
#include "aqsgd_adamw.h"
#include "aqsgd_layernorm.h"

namespace aqsgd {
namespace {

constexpr int kLanes = 256;

__device__ __forceinline__ double workgroup_sum(double v, double* part) {
    v = lanes_sum<kWave>(v);
    if ((threadIdx.x & (kWave - 1)) == 0) part[threadIdx.x / kWave] = v;
    __syncthreads();
    return part[0] + part[1] + part[2] + part[3];
}

template <int GT>
__global__ __launch_bounds__(kLanes) void grad_squares_kernel(const NormTable table, const int64_t span, double* partial) {
    __shared__ double part[4];
    const int which = __builtin_amdgcn_readfirstlane(__popcll(__ballot(table.first[threadIdx.x & (kWave - 1)] <= blockIdx.x)) - 1);
    const int64_t n = table.n[which], begin = static_cast<int64_t>(blockIdx.x - table.first[which]) * span;
    const int64_t end = begin + span < n ? begin + span : n;
    double sum = 0.0;
    for (int64_t i = begin + threadIdx.x * 4; i < end; i += kLanes * 4) {
        float f[4];
        load_four<GT, false>(table.grad[which], i, end - i < 4 ? static_cast<int>(end - i) : 4, f);
#pragma unroll
        for (int e = 0; e < 4; ++e) sum = fma(static_cast<double>(f[e]), static_cast<double>(f[e]), sum);
    }
    sum = workgroup_sum(sum, part);
    if (threadIdx.x == 0) partial[blockIdx.x] = sum;
}

__global__ __launch_bounds__(kLanes) void grad_norm_kernel(const double* partial, const int64_t count, const double max_norm, const float* loss_scale, float* result) {
    __shared__ double part[4];
    double sum = 0.0;
    for (int64_t i = threadIdx.x; i < count; i += kLanes) sum += partial[i];
    sum = workgroup_sum(sum, part);
    if (threadIdx.x != 0) return;
    const double inverse = loss_scale ? 1.0 / static_cast<double>(*loss_scale) : 1.0, norm = sqrt(sum) * inverse;
    const double clip = max_norm / norm;                    // 0 / 0, of no gradient at all: nothing to clip
    result[0] = static_cast<float>(norm);
    result[1] = norm < __builtin_inf() ? static_cast<float>((clip < 1.0 ? clip : 1.0) * inverse) : __builtin_nanf("");
}

}  // namespace

hipError_t launch_grad_squares(int dtype, const NormTable& table, uint32_t blocks, int64_t span, double* partial, hipStream_t stream) {
    const dim3 grid(blocks), block(kLanes);
    switch (dtype) {
    case AQSGD_F32:  return launch_kernel(grad_squares_kernel<AQSGD_F32>, grid, block, stream, table, span, partial);
    case AQSGD_F16:  return launch_kernel(grad_squares_kernel<AQSGD_F16>, grid, block, stream, table, span, partial);
    default:         return launch_kernel(grad_squares_kernel<AQSGD_BF16>, grid, block, stream, table, span, partial);
    }
}

hipError_t launch_grad_norm(const double* partial, int64_t count, double max_norm, const float* loss_scale, float* result, hipStream_t stream) {
    return launch_kernel(grad_norm_kernel, dim3(1), dim3(kLanes), stream, partial, count, max_norm, loss_scale, result);
}

}  // namespace aqsgd
