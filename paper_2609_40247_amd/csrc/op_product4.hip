// Products of rows with 4-bit weights: the entry points, and the kernels for bf16 rows.
#include "product4.hpp"

namespace hop {
int product_bf16(ProductArgs& p) { return product_group<HERSCHEL_BF16, false>(p); }
}  // namespace hop

extern "C" int herschel_product4_workspace(int64_t n_rows, int32_t kind, int32_t gated, int32_t n, int32_t k, size_t* bytes) {
  using namespace hop;
  if (!bytes || n_rows < 0 || kind < HERSCHEL_BF16 || kind > HERSCHEL_INT8 || n < 1 || n > HERSCHEL_MAX_WEIGHT_ROWS || k < 1 ||
      k > (1 << 30))
    return HERSCHEL_EINVAL;
  ProductArgs p{};
  p.a.n_rows = n_rows;
  p.a.kind = kind;
  p.a.gated = gated;
  p.tiles_n = (n + 15) / 16;
  p.tiles_k = (k + 127) / 128;
  p.half = n / 32;
  const int splits = n_rows == 0 ? 1 : choose(p, SIZE_MAX).splits;
  *bytes = splits > 1 ? parts_bytes(p, splits) : 0;
  return HERSCHEL_OK;
}

extern "C" int herschel_product4(const herschel_product_args* args, const herschel_weights4* weights) {
  using namespace hop;
  if (!args || !weights) return HERSCHEL_EINVAL;
  const herschel_product_args& a = *args;
  const herschel_weights4& w = *weights;
  if (w.n < 1 || w.k < 1 || (w.group != 32 && w.group != 64 && w.group != 128))
    return HERSCHEL_EINVAL;
  // k with what a phase reads beyond stays in 31 bits; the threads of the largest n's workgroups, each 768 for 8 tiles of
  // 16 rows, in the 32 that a launch counts them in
  if (w.k > (1 << 30) || w.n > HERSCHEL_MAX_WEIGHT_ROWS) return HERSCHEL_EINVAL;
  if (!w.codes || !w.scales || !aligned(w.codes, 16) || !aligned(w.scales, 16))
    return HERSCHEL_EINVAL;
  if (!type_ok(a.type) || (a.kind != a.type && !quantised(a.kind)) || a.x_row < 0) return HERSCHEL_EINVAL;
  if (a.n_rows < 0 || a.n_rows > HERSCHEL_MAX_PRODUCT_ROWS) return HERSCHEL_EINVAL;
  if (a.x_group && (!quantised(a.kind) || a.x_group != w.group)) return HERSCHEL_EINVAL;
  if (a.gated && w.n % 32) return HERSCHEL_EINVAL;
  if (a.n_rows == 0) return HERSCHEL_OK;  // nothing to point at
  if (!a.x || !a.out || !aligned(a.out, 2) || !aligned(a.x, quantised(a.kind) ? 1 : 2)) return HERSCHEL_EINVAL;
  if (quantised(a.kind) && (!a.x_scale || !aligned(a.x_scale, 4))) return HERSCHEL_EINVAL;
  // a row of x and a tile of the weights are read by many workgroups, some after others have written
  const int64_t e = quantised(a.kind) ? 1 : 2, groups = a.x_group ? (w.k + w.group - 1) / w.group : 1;
  const int64_t tiles = (int64_t)((w.k + 127) / 128) * ((w.n + 15) / 16), row = (int64_t)(a.gated ? w.n / 2 : w.n) * 2;
  const RowsMemory out{a.out, a.n_rows, row, row};
  if (share_memory(out, {a.x, a.n_rows, a.x_row * e, w.k * e})) return HERSCHEL_EINVAL;
  if (quantised(a.kind) && share_memory(out, {a.x_scale, a.n_rows, groups * 4, groups * 4})) return HERSCHEL_EINVAL;
  if (share_memory(out, {w.codes, tiles, 1024, 1024}) || share_memory(out, {w.scales, tiles, 8192 / w.group, 8192 / w.group}))
    return HERSCHEL_EINVAL;
  ProductArgs p{};
  p.a = a;
  p.w = w;
  p.tiles_k = (w.k + 127) / 128;
  p.tiles_n = (w.n + 15) / 16;
  p.half = w.n / 32;
  switch (a.kind) {
    case HERSCHEL_FP8: return a.x_group ? product_fp8_groups(p) : product_fp8(p);
    case HERSCHEL_INT8: return a.x_group ? product_int8_groups(p) : product_int8(p);
    case HERSCHEL_BF16: return product_bf16(p);
    default: return product_f16(p);
  }
}
