// Tiles of 8-bit products with float32 results.
#include "aqsgd_matmul8.h"

namespace aqsgd {
template hipError_t launch_product_dt<AQSGD_F32>(ProductTile, ProductKind, const ProductArgs&, hipStream_t);
}
