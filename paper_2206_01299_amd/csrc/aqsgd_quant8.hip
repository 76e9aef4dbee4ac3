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

hipError_t launch_quant8(int dtype, int rounding, const Quant8Args& a, hipStream_t stream) {
    const bool draw = rounding == AQSGD_ROUND_STOCHASTIC;
    switch (dtype) {
    case AQSGD_F32:  return draw ? launch_quant8_as<AQSGD_F32, 1>(a, stream) : launch_quant8_as<AQSGD_F32, 0>(a, stream);
    case AQSGD_F16:  return draw ? launch_quant8_as<AQSGD_F16, 1>(a, stream) : launch_quant8_as<AQSGD_F16, 0>(a, stream);
    default:         return draw ? launch_quant8_as<AQSGD_BF16, 1>(a, stream) : launch_quant8_as<AQSGD_BF16, 0>(a, stream);
    }
}

}  // namespace aqsgd
