// Products of rows with 4-bit weights: the kernels for fp8 rows with a scale for each group.
#include "product4.hpp"

namespace hop {
int product_fp8_groups(ProductArgs& p) { return product_group<HERSCHEL_FP8, true>(p); }
}  // namespace hop
