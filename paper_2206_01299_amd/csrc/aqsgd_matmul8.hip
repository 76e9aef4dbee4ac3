// Products of 8-bit codes: which kernel a call takes.
#include "aqsgd_matmul8.h"

namespace aqsgd {

extern template hipError_t launch_product_dt<AQSGD_F32>(ProductTile, ProductKind, const ProductArgs&, hipStream_t);
extern template hipError_t launch_product_dt<AQSGD_F16>(ProductTile, ProductKind, const ProductArgs&, hipStream_t);
extern template hipError_t launch_product_dt<AQSGD_BF16>(ProductTile, ProductKind, const ProductArgs&, hipStream_t);

namespace {
ProductTile choose_tile(ProductKind kind, const ProductArgs& p) {
    const int64_t size = static_cast<int64_t>(p.m) * p.n;
    if (size >= 256 * 256 * 128) return kTile256;
    if (p.m <= 16) return kind == kGated ? kSplit16x32 : kSplit16;
    if (p.m <= 32) return kSplit32;
    if (size >= 64 * 64 * 512) return kTile128;
    return kSplit64;
}
}  // namespace

hipError_t launch_product(ProductKind kind, const ProductArgs& p, hipStream_t stream) {
    const ProductTile tile = choose_tile(kind, p);
    switch (p.dtype) {
    case AQSGD_F32:  return launch_product_dt<AQSGD_F32>(tile, kind, p, stream);
    case AQSGD_F16:  return launch_product_dt<AQSGD_F16>(tile, kind, p, stream);
    default:         return launch_product_dt<AQSGD_BF16>(tile, kind, p, stream);
    }
}

}  // namespace aqsgd
