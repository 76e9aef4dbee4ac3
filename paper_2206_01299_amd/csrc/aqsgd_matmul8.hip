// Products of 8-bit codes: which kernel a call takes.
#include "aqsgd_matmul8.h"

namespace aqsgd {

hipError_t launch_product(ProductKind kind, const ProductArgs& p, hipStream_t stream) {
    const int64_t tiles = ((p.m + 63) / 64) * static_cast<int64_t>((p.n + 63) / 64);
    const dim3 grid(static_cast<unsigned>(tiles)), block(256);
    switch (kind) {
    case kPlain:      return launch_kernel(product64_kernel<kPlain>, grid, block, stream, p);
    case kMessage:    return launch_kernel(product64_kernel<kMessage>, grid, block, stream, p);
    case kActivation: return launch_kernel(product64_kernel<kActivation>, grid, block, stream, p);
    default:          return launch_kernel(product64_kernel<kGated>, grid, block, stream, p);
    }
}

}  // namespace aqsgd
