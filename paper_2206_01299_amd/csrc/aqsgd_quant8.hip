// Signed 8-bit codes: which kernels a call takes.
#include "aqsgd_quant8.h"

namespace aqsgd {

int64_t quant8_workspace_bytes(int64_t rows, int64_t cols) { return rows > 0 && cols > 0 ? col_blocks(rows) * cols * 8 : 0; }

hipError_t launch_quant8(int dtype, int rounding, const Quant8Args& a, hipStream_t stream) {
    const bool draw = rounding == AQSGD_ROUND_STOCHASTIC;
    switch (dtype) {
    case AQSGD_F32:  return draw ? launch_quant8_as<AQSGD_F32, 1>(a, stream) : launch_quant8_as<AQSGD_F32, 0>(a, stream);
    case AQSGD_F16:  return draw ? launch_quant8_as<AQSGD_F16, 1>(a, stream) : launch_quant8_as<AQSGD_F16, 0>(a, stream);
    default:         return draw ? launch_quant8_as<AQSGD_BF16, 1>(a, stream) : launch_quant8_as<AQSGD_BF16, 0>(a, stream);
    }
}

}  // namespace aqsgd
