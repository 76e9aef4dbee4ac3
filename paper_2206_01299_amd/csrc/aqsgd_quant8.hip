// Signed 8-bit codes: the types' kernels, and the workspace of the columns'.
#include "aqsgd_quant8.h"

namespace aqsgd {

#define AQSGD_EXTERN_QUANT8(DT)                                                                                 \
    extern template hipError_t launch_quant8_as<DT, AQSGD_ROUND_NEAREST>(const Quant8Args&, hipStream_t);       \
    extern template hipError_t launch_quant8_as<DT, AQSGD_ROUND_STOCHASTIC>(const Quant8Args&, hipStream_t);
AQSGD_EXTERN_QUANT8(AQSGD_F32)
AQSGD_EXTERN_QUANT8(AQSGD_F16)
AQSGD_EXTERN_QUANT8(AQSGD_BF16)

int64_t quant8_workspace_bytes(int64_t rows, int64_t cols) {
    if (rows <= 0 || cols <= 0) return 0;
    const ColumnPlan p = column_plan(rows, cols);
    return (2 * p.blocks * cols + p.spans * rows) * 4;
}

// Vectors of no elements: scale 0 and sum 0, so that a product over no tokens is 0.
static __global__ __launch_bounds__(256) void quant8_empty_kernel(float* scales, float* sums, int64_t count) {
    for (int64_t i = blockIdx.x * int64_t{256} + threadIdx.x; i < count; i += int64_t{256} * gridDim.x) {
        if (scales) scales[i] = 0.0f;
        if (sums) sums[i] = 0.0f;
    }
}

hipError_t launch_quant8_empty(float* scales, float* sums, int64_t count, hipStream_t stream) {
    const int64_t blocks = (count + 255) / 256;
    return launch_kernel(quant8_empty_kernel, dim3(static_cast<unsigned>(blocks < 4096 ? blocks : 4096)), dim3(256), stream, scales, sums, count);
}

hipError_t launch_quant8(int dtype, int rounding, const Quant8Args& a, hipStream_t stream) {
    const bool draw = rounding == AQSGD_ROUND_STOCHASTIC;
    switch (dtype) {
    case AQSGD_F32:  return draw ? launch_quant8_as<AQSGD_F32, 1>(a, stream) : launch_quant8_as<AQSGD_F32, 0>(a, stream);
    case AQSGD_F16:  return draw ? launch_quant8_as<AQSGD_F16, 1>(a, stream) : launch_quant8_as<AQSGD_F16, 0>(a, stream);
    default:         return draw ? launch_quant8_as<AQSGD_BF16, 1>(a, stream) : launch_quant8_as<AQSGD_BF16, 0>(a, stream);
    }
}

}  // namespace aqsgd
