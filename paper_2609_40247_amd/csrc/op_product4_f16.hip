// Products of rows with 4-bit weights: the kernels for half rows.
#include "product4.hpp"

namespace hop {
int product_f16(ProductArgs& p) { return product_group<HERSCHEL_F16, false>(p); }
}  // namespace hop
