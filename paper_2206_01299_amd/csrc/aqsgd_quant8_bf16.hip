// Signed 8-bit codes of bfloat16 matrices.
#include "aqsgd_quant8.h"

namespace aqsgd {
template hipError_t launch_quant8_as<AQSGD_BF16, AQSGD_ROUND_NEAREST>(const Quant8Args&, hipStream_t);
template hipError_t launch_quant8_as<AQSGD_BF16, AQSGD_ROUND_STOCHASTIC>(const Quant8Args&, hipStream_t);
}
