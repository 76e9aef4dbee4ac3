// AdamW: the step's kernels for each type of weights and gradients.
#include "aqsgd_adamw.h"

namespace aqsgd {

int64_t adamw_workgroups(int64_t n) { return (n + kUpdateSpan - 1) / kUpdateSpan; }

hipError_t launch_adamw(const AdamwKind& kind, const UpdateTable& table, uint32_t blocks, const AdamwArgs& a, hipStream_t stream) {
    const bool wide = kind.grad_dtype == AQSGD_F32;
    switch (kind.dtype) {
    case AQSGD_F32:  return launch_adamw_as<AQSGD_F32, AQSGD_F32>(kind, table, blocks, a, stream);
    case AQSGD_F16:  return wide ? launch_adamw_as<AQSGD_F16, AQSGD_F32>(kind, table, blocks, a, stream)
                                 : launch_adamw_as<AQSGD_F16, AQSGD_F16>(kind, table, blocks, a, stream);
    default:         return wide ? launch_adamw_as<AQSGD_BF16, AQSGD_F32>(kind, table, blocks, a, stream)
                                 : launch_adamw_as<AQSGD_BF16, AQSGD_BF16>(kind, table, blocks, a, stream);
    }
}

}  // namespace aqsgd
