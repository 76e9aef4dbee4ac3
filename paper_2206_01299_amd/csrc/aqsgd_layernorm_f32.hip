// Layer norm of binary32 rows, and its gradient.
#include "aqsgd_layernorm.h"

namespace aqsgd {
template hipError_t launch_layernorm_as<AQSGD_F32>(const LayernormArgs&, hipStream_t);
template hipError_t launch_layernorm_grad_as<AQSGD_F32>(const LayernormGradArgs&, hipStream_t);
}
