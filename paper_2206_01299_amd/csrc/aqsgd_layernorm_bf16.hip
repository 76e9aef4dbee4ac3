// Layer norm of bfloat16 rows, and its gradient.
#include "aqsgd_layernorm.h"

namespace aqsgd {
template hipError_t launch_layernorm_as<AQSGD_BF16>(const LayernormArgs&, hipStream_t);
template hipError_t launch_layernorm_grad_as<AQSGD_BF16>(const LayernormGradArgs&, hipStream_t);
}
