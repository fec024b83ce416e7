// Products of rows with 4-bit weights: the kernels for int8 rows.
#include "product4.hpp"

namespace hop {
int product_int8(ProductArgs& p) { return product_group<HERSCHEL_INT8, false>(p); }
}  // namespace hop
