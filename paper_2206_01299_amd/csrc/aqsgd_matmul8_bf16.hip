// 8-bit products with bfloat16 results.
#include "aqsgd_matmul8.h"

namespace aqsgd {
AQSGD_PRODUCT_DT(, AQSGD_BF16)
}
