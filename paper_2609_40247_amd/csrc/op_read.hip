// The paged cache read back as dense rows: every code and scale read once,
// every element written once, nothing computed but the scaling.  Bound by the
// traffic: 717 MB of int8 rows to half in 142 us, 5.1 TB/s, the rate of a copy (on
// some cards 132 us).
#include "ops.hpp"

namespace hop {

struct ReadArgs {
  herschel_read_args a;
  herschel_cache c;
  int page_shift;
  int parts;  // workgroups that share a token's heads
};

// A group of G lanes (head_dim / 16 rounded up to a power of two) takes one
// token, 16 elements a lane, and walks its heads, keys and values: the
// sequence and page of the token are found once for all of them, and
// neighbouring groups read neighbouring rows of a page.
template <int TYPE, int KIND, int G>
__global__ __launch_bounds__(256) void k_cache_read(ReadArgs p) {
  const herschel_read_args& a = p.a;
  const int lane = threadIdx.x % G, D = p.c.head_dim, heads = p.c.n_heads;
  const int part = blockIdx.x % p.parts;
  const int64_t t = (int64_t)(blockIdx.x / p.parts) * (256 / G) + threadIdx.x / G;
  if (t >= a.n_rows || lane * 16 >= D) return;
  int lo = 0, hi = a.n_seqs;  // the last sequence that starts at or before t
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (a.cu[mid] <= t) lo = mid;
    else hi = mid;
  }
  const int64_t at = t - a.cu[lo], entry = at >> p.page_shift;
  const bool in_row = at >= 0 && t < a.cu[lo + 1] && entry < a.table_stride;
  int64_t page = in_row ? a.block_table[lo * a.table_stride + entry] : 0;
  const bool good = in_row && page >= 0 && page < p.c.n_pages;
  if (!good) {
    page = 0;
    if (lane == 0 && part == 0) flag(a.status, in_row ? HERSCHEL_OP_BAD_PAGE : HERSCHEL_OP_BAD_LENGTH);
  }
  const int64_t row0 = ((page * heads) << p.page_shift) + (at & (p.c.page_size - 1));
  // HB heads' rows are asked for before the first is waited for
  constexpr int HB = 4, W = quantised(KIND) ? 1 : 2;
  for (int h0 = part; h0 < heads; h0 += HB * p.parts) {
    u32x4 x[HB][2][W];
    float scale[HB][2];
#pragma unroll
    for (int i = 0; i < HB; ++i) {
      const int h = h0 + i * p.parts;
      const int64_t row = row0 + ((int64_t)h << p.page_shift);
#pragma unroll
      for (int v = 0; v < 2; ++v) {
#pragma unroll
        for (int w = 0; w < W; ++w) x[i][v][w] = u32x4{0, 0, 0, 0};
        scale[i][v] = 0;
        if (!good || h >= heads || !(v ? a.v_out : a.k_out)) continue;
        const u32x4* src = (const u32x4*)((const char*)(v ? p.c.v : p.c.k) + (row * D + lane * 16) * code_bytes(KIND));
#pragma unroll
        for (int w = 0; w < W; ++w) x[i][v][w] = src[w];
        if constexpr (quantised(KIND)) scale[i][v] = (v ? p.c.v_scale : p.c.k_scale)[row];
      }
    }
#pragma unroll
    for (int i = 0; i < HB; ++i) {
      const int h = h0 + i * p.parts;
#pragma unroll
      for (int v = 0; v < 2; ++v) {
        uint16_t* out = (uint16_t*)(v ? a.v_out : a.k_out);
        if (h >= heads || !out) continue;
        u32x4 w[2];
        if constexpr (!quantised(KIND)) {
          w[0] = x[i][v][0];
          w[1] = x[i][v][1];
        } else {
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            float e[4];
            decode2f<KIND, false>(x[i][v][0][j], e[0], e[1]);
            decode2f<KIND, true>(x[i][v][0][j], e[2], e[3]);
            w[j / 2][2 * (j & 1)] = pack2<TYPE>(e[0] * scale[i][v], e[1] * scale[i][v]);
            w[j / 2][2 * (j & 1) + 1] = pack2<TYPE>(e[2] * scale[i][v], e[3] * scale[i][v]);
          }
        }
        u32x4* dst = (u32x4*)(out + (t * heads + h) * D + lane * 16);
        dst[0] = w[0];
        dst[1] = w[1];
      }
    }
  }
}

template <int TYPE, int KIND>
static int read_launch(ReadArgs& p) {
  const int G = p.c.head_dim <= 64 ? 4 : p.c.head_dim <= 128 ? 8 : 16, per = 256 / G;
  const int64_t tiles = (p.a.n_rows + per - 1) / per;
  // enough workgroups to fill 256 CUs a few times over, by splitting the heads
  p.parts = 1;
  while (p.parts < p.c.n_heads && tiles * p.parts < 2048) p.parts *= 2;
  if (p.parts > p.c.n_heads) p.parts = p.c.n_heads;
  if (tiles * p.parts > 0x7fffffff) return HERSCHEL_EINVAL;
  void (*k)(ReadArgs) = G == 4   ? k_cache_read<TYPE, KIND, 4>
                        : G == 8 ? k_cache_read<TYPE, KIND, 8>
                                 : k_cache_read<TYPE, KIND, 16>;
  // Large reads run with five workgroups a CU at most, by LDS that nobody uses:
  // fewer rows under way at once, in longer runs, suit the memory better (717 MB
  // 142 against 162 us, 497 MB 111 against 117); small ones want all there are
  // (34 MB 10.2 against 11.0 us).
  const bool large = p.a.n_rows * p.c.n_heads * p.c.head_dim >= (16 << 20);
  return launch(k, dim3((unsigned)(tiles * p.parts)), dim3(256), large ? 32768 : 0, p.a.hip_stream, p);
}

}  // namespace hop

extern "C" int herschel_cache_read(const herschel_read_args* args, const herschel_cache* cache) {
  using namespace hop;
  if (!args || !cache_ok(cache) || cache->head_dim % 16) return HERSCHEL_EINVAL;
  const herschel_read_args& a = *args;
  if (a.n_seqs < 1 || a.n_rows < 0 || a.table_stride < 0 || !a.cu || !type_ok(a.type)) return HERSCHEL_EINVAL;
  if (a.n_rows > 0x7fffffff || (!a.block_table && a.table_stride)) return HERSCHEL_EINVAL;
  if ((a.k_out && !aligned(a.k_out, 16)) || (a.v_out && !aligned(a.v_out, 16))) return HERSCHEL_EINVAL;
  if (!quantised(cache->kind) && cache->kind != a.type) return HERSCHEL_EINVAL;
  if (a.n_rows == 0 || (!a.k_out && !a.v_out)) return HERSCHEL_OK;
  ReadArgs p{a, *cache, log2i(cache->page_size), 1};
  const bool bf = a.type == HERSCHEL_BF16;
  switch (cache->kind) {
    case HERSCHEL_FP8:
      return bf ? read_launch<HERSCHEL_BF16, HERSCHEL_FP8>(p) : read_launch<HERSCHEL_F16, HERSCHEL_FP8>(p);
    case HERSCHEL_INT8:
      return bf ? read_launch<HERSCHEL_BF16, HERSCHEL_INT8>(p) : read_launch<HERSCHEL_F16, HERSCHEL_INT8>(p);
    default:
      return bf ? read_launch<HERSCHEL_BF16, HERSCHEL_BF16>(p) : read_launch<HERSCHEL_F16, HERSCHEL_F16>(p);
  }
}
