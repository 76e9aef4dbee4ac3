// Products of 8-bit codes: which kernel a call takes.
#include "aqsgd_matmul8.h"

namespace aqsgd {

extern template hipError_t launch_product_dt<AQSGD_F32>(ProductTile, ProductKind, const ProductArgs&, hipStream_t);
extern template hipError_t launch_product_dt<AQSGD_F16>(ProductTile, ProductKind, const ProductArgs&, hipStream_t);
extern template hipError_t launch_product_dt<AQSGD_BF16>(ProductTile, ProductKind, const ProductArgs&, hipStream_t);

hipError_t launch_product(ProductKind kind, const ProductArgs& p, hipStream_t stream) {
    const ProductTile tile = static_cast<int64_t>(p.m) * p.n >= 256 * 256 * 128 ? kTile256 : kTile128;
    switch (p.dtype) {
    case AQSGD_F32:  return launch_product_dt<AQSGD_F32>(tile, kind, p, stream);
    case AQSGD_F16:  return launch_product_dt<AQSGD_F16>(tile, kind, p, stream);
    default:         return launch_product_dt<AQSGD_BF16>(tile, kind, p, stream);
    }
}

}  // namespace aqsgd
