// Products of rows with 4-bit weights: the kernels for int8 rows with a scale for each group.
#include "product4.hpp"

namespace hop {
int product_int8_groups(ProductArgs& p) { return product_group<HERSCHEL_INT8, true>(p); }
}  // namespace hop
