// 8-bit products with float32 results.
#include "aqsgd_matmul8.h"

namespace aqsgd {
AQSGD_PRODUCT_DT(, AQSGD_F32)
}
