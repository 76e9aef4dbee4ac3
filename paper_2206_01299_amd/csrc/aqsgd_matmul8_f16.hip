// Tiles of 8-bit products with float16 results.
#include "aqsgd_matmul8.h"

namespace aqsgd {
template hipError_t launch_product_dt<AQSGD_F16>(ProductTile, ProductKind, const ProductArgs&, hipStream_t);
}
