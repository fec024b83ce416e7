// Products of rows with 4-bit weights: the kernels for fp8 rows.
#include "product4.hpp"

namespace hop {
int product_fp8(ProductArgs& p) { return product_group<HERSCHEL_FP8, false>(p); }
}  // namespace hop
