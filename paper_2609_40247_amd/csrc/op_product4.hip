// Products of a few rows with 4-bit weights, one launch.
//
// y[m][n] = sum_g s[n][g] (sum_{k in g} c[n][k] x[m][k] - z[n][g] sum_{k in g} x[m][k]).
// The codes enter the matrix cores as what they are, 0 to 15: as bytes they are
// whole numbers, and read as fp8 they are c 2^-9 exactly (0 to 7 as its
// subnormals, 8 to 15 as its first eight normals), so fp8 rows meet them as they
// are and 16-bit rows after a conversion of fp8 pairs, which has an instruction.
// The group's sum of x, which the zero needs, comes from one more product with a
// constant operand; scale and zero meet the group's sums, not the weights.
// The bytes of the weights bound it: every code is read once, in runs of 1 KB a
// wave, and nothing of it is written back.
#include "ops.hpp"

namespace hop {

struct ProductArgs {
  herschel_product_args a;
  herschel_weights4 w;
  int tiles_k;   // tiles of 128 columns
  int half;      // gated: tiles of 16 rows from a row to the one it gates
};

typedef u32x4 u32x4_any __attribute__((aligned(1)));
typedef u32x2 u32x2_any __attribute__((aligned(1)));
typedef int i32x4 __attribute__((ext_vector_type(4)));

template <int KIND> struct Sum { typedef f32x4 T; };
template <> struct Sum<HERSCHEL_INT8> { typedef i32x4 T; };
template <int KIND> struct Operand { typedef u32x4 T; };  // eight elements
template <> struct Operand<HERSCHEL_FP8> { typedef u32x2 T; };
template <> struct Operand<HERSCHEL_INT8> { typedef u32x2 T; };

// D += A B of 32 columns: A the weights, 16 rows, B sixteen rows of x.
template <int KIND>
__device__ __forceinline__ typename Sum<KIND>::T mma(typename Operand<KIND>::T a, typename Operand<KIND>::T b,
                                                     typename Sum<KIND>::T c) {
  if constexpr (KIND == HERSCHEL_FP8)
    return __builtin_amdgcn_mfma_f32_16x16x32_fp8_fp8(__builtin_bit_cast(long, a), __builtin_bit_cast(long, b), c, 0, 0, 0);
  else if constexpr (KIND == HERSCHEL_INT8)
    return __builtin_amdgcn_mfma_i32_16x16x32_i8(__builtin_bit_cast(long, a), __builtin_bit_cast(long, b), c, 0, 0, 0);
  else return mfma16<KIND>(a, b, c);
}

// A word's eight codes as an operand: byte b holds columns b and b + 4.
template <int KIND>
__device__ __forceinline__ typename Operand<KIND>::T unpack_codes(uint32_t w) {
  const uint32_t lo = w & 0x0f0f0f0fu, hi = (w >> 4) & 0x0f0f0f0fu;
  if constexpr (quantised(KIND)) return u32x2{lo, hi};
  else
    return u32x4{decode2<HERSCHEL_FP8, KIND, false>(lo), decode2<HERSCHEL_FP8, KIND, true>(lo),
                 decode2<HERSCHEL_FP8, KIND, false>(hi), decode2<HERSCHEL_FP8, KIND, true>(hi)};
}
// Ones in the codes' unit, in every place.
template <int KIND>
__device__ __forceinline__ typename Operand<KIND>::T ones() {
  if constexpr (quantised(KIND)) return u32x2{0x01010101u, 0x01010101u};
  else {
    const uint32_t one = decode2<HERSCHEL_FP8, KIND, false>(0x0101u);
    return u32x4{one, one, one, one};
  }
}

// Eight elements of a row of x from column k on; those from column K on are 0.
template <int KIND>
__device__ __forceinline__ typename Operand<KIND>::T load_x(const void* x, int64_t at, int k, int K) {
  if constexpr (quantised(KIND)) {
    const uint8_t* p = (const uint8_t*)x + at + k;
    if (k + 8 <= K) return *(const u32x2_any*)p;
    u32x2 r = {0, 0};
    for (int i = 0; i < 8; ++i)
      if (k + i < K) r[i / 4] |= (uint32_t)p[i] << (8 * (i % 4));
    return r;
  } else {
    const uint16_t* p = (const uint16_t*)x + at + k;
    if (k + 8 <= K) return *(const u32x4_any*)p;
    u32x4 r = {0, 0, 0, 0};
    for (int i = 0; i < 8; ++i)
      if (k + i < K) r[i / 2] |= (uint32_t)p[i] << (16 * (i % 2));
    return r;
  }
}

template <int TYPE>
__device__ __forceinline__ float scale_of(uint32_t bits) {
  float a, unused;
  unpack2<TYPE>(bits & 0xffffu, a, unused);
  return a;
}

// A workgroup takes NT tiles of 16 weight rows (gated: half of them of the rows
// that gate, half of those that they gate) and up to 16 MT rows of x; its waves
// share the columns, 128 at a time, and their sums meet in LDS.
template <int KIND, int TYPE, int GROUP, int MT, int NT>
__global__ __launch_bounds__(512) void k_product4(ProductArgs p) {
  const herschel_product_args& a = p.a;
  const herschel_weights4& w = p.w;
  constexpr int PER = 128 / GROUP, STEPS = GROUP / 32;
  typedef typename Sum<KIND>::T SumT;
  typedef typename Operand<KIND>::T Op;
  extern __shared__ f32x4 parts[];
  const int lane = threadIdx.x % WAVE, wave = threadIdx.x / WAVE, waves = blockDim.x / WAVE;
  const int q = lane / 16, col = lane % 16;
  const int64_t m0 = (int64_t)blockIdx.y * (16 * MT);
  const int K = w.k, groups = (K + GROUP - 1) / GROUP;
  const bool gated = a.gated != 0;
  int tile[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t)
    tile[t] = gated ? (int)blockIdx.x * (NT / 2) + t % (NT / 2 > 0 ? NT / 2 : 1) + (t >= NT / 2 ? p.half : 0)
                    : (int)blockIdx.x * NT + t;
  const int tiles_n = (w.n + 15) / 16, last_n = gated ? p.half : tiles_n;
  int64_t row[MT];  // rows beyond the last are computed as it and not stored
#pragma unroll
  for (int t = 0; t < MT; ++t) row[t] = min(m0 + 16 * t + col, a.n_rows - 1);
  f32x4 sum[MT][NT];
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int t = 0; t < NT; ++t) sum[i][t] = f32x4{0, 0, 0, 0};

  for (int kt = wave; kt < p.tiles_k; kt += waves) {
    u32x4 code[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      const int at = min(tile[t], tiles_n - 1);
      code[t] = *((const u32x4*)w.codes + ((int64_t)at * p.tiles_k + kt) * WAVE + lane);
    }
    Op x[MT][4];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) x[i][j] = load_x<KIND>(a.x, row[i] * a.x_row, kt * 128 + 32 * j + 8 * q, K);
#pragma unroll
    for (int g = 0; g < PER; ++g) {
      SumT of_x[MT];
#pragma unroll
      for (int i = 0; i < MT; ++i) {
        of_x[i] = SumT{0, 0, 0, 0};
#pragma unroll
        for (int j = 0; j < STEPS; ++j) of_x[i] = mma<KIND>(ones<KIND>(), x[i][g * STEPS + j], of_x[i]);
      }
      float xs[MT];
#pragma unroll
      for (int i = 0; i < MT; ++i)
        xs[i] = quantised(KIND) && a.x_group && kt * PER + g < groups ? a.x_scale[row[i] * groups + kt * PER + g] : 1.0f;
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        const int64_t at = ((int64_t)min(tile[t], tiles_n - 1) * p.tiles_k * PER + kt * PER + g) * 16 + 4 * q;
        const u32x2 s2 = *(const u32x2*)((const uint16_t*)w.scales + at);
        const uint32_t z4 = w.zeros ? *(const uint32_t*)(w.zeros + at) : 0x08080808u;
        float s[4], z[4];
        if (w.scale_type == HERSCHEL_BF16) {
          unpack2<HERSCHEL_BF16>(s2[0], s[0], s[1]);
          unpack2<HERSCHEL_BF16>(s2[1], s[2], s[3]);
        } else {
          unpack2<HERSCHEL_F16>(s2[0], s[0], s[1]);
          unpack2<HERSCHEL_F16>(s2[1], s[2], s[3]);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) z[i] = (float)((z4 >> (8 * i)) & 0xffu);
        Op codes[STEPS];
#pragma unroll
        for (int j = 0; j < STEPS; ++j) codes[j] = unpack_codes<KIND>(code[t][g * STEPS + j]);
#pragma unroll
        for (int i = 0; i < MT; ++i) {
          SumT d = {0, 0, 0, 0};
#pragma unroll
          for (int j = 0; j < STEPS; ++j) d = mma<KIND>(codes[j], x[i][g * STEPS + j], d);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float y = ((float)d[e] - z[e] * (float)of_x[i][e]) * s[e];
            sum[i][t][e] += quantised(KIND) ? y * xs[i] : y;
          }
        }
      }
    }
  }

#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int t = 0; t < NT; ++t) parts[((wave * MT + i) * NT + t) * WAVE + lane] = sum[i][t];
  __syncthreads();
  const int outs = gated ? NT / 2 : NT, n_out = gated ? w.n / 2 : w.n;
  for (int o = threadIdx.x; o < MT * outs * WAVE; o += blockDim.x) {
    const int l = o % WAVE, t = o / WAVE % outs, i = o / WAVE / outs;
    const int64_t m = m0 + 16 * i + l % 16;
    const int at = (int)blockIdx.x * outs + t;
    const int n = 16 * at + 4 * (l / 16);
    if (m >= a.n_rows || at >= last_n || n >= n_out) continue;
    f32x4 y = {0, 0, 0, 0}, b = {0, 0, 0, 0};
    for (int v = 0; v < waves; ++v) {
      y += parts[((v * MT + i) * NT + t) * WAVE + l];
      if (gated) b += parts[((v * MT + i) * NT + t + outs) * WAVE + l];
    }
    float by = KIND == HERSCHEL_INT8 ? 1.0f : 512.0f;
    if (quantised(KIND) && !a.x_group) by *= a.x_scale[m];
    y *= by;
    if (gated) {
      b *= by;
#pragma unroll
      for (int e = 0; e < 4; ++e) y[e] = y[e] / (1.0f + expf(-y[e])) * b[e];
    }
    const uint32_t w0 = pack2<TYPE>(y[0], y[1]), w1 = pack2<TYPE>(y[2], y[3]);
    uint16_t* to = (uint16_t*)a.out + m * n_out + n;
    if (n_out % 4 == 0 && ((uintptr_t)a.out & 7) == 0) {
      *(u32x2*)to = u32x2{w0, w1};
    } else {
      const uint16_t h[4] = {(uint16_t)w0, (uint16_t)(w0 >> 16), (uint16_t)w1, (uint16_t)(w1 >> 16)};
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (n + e < n_out) to[e] = h[e];
    }
  }
}

template <int KIND, int TYPE, int GROUP, int MT, int NT>
static int product_launch(ProductArgs& p) {
  const int tiles = p.a.gated ? p.half * 2 : (p.w.n + 15) / 16;
  const int64_t blocks = (p.a.n_rows + 16 * MT - 1) / (16 * MT);
  if (blocks > 65535) return HERSCHEL_EINVAL;
  int waves = 8;
  while (waves > 1 && waves > p.tiles_k) waves /= 2;
  return launch(k_product4<KIND, TYPE, GROUP, MT, NT>, dim3((unsigned)((tiles + NT - 1) / NT), (unsigned)blocks),
                dim3(waves * WAVE), (size_t)waves * MT * NT * WAVE * sizeof(f32x4), p.a.hip_stream, p);
}
template <int KIND, int TYPE, int GROUP>
static int product_tiles(ProductArgs& p) {
  if (p.a.n_rows <= 16) return product_launch<KIND, TYPE, GROUP, 1, 2>(p);
  if (p.a.n_rows <= 32) return product_launch<KIND, TYPE, GROUP, 2, 2>(p);
  return product_launch<KIND, TYPE, GROUP, 4, 2>(p);
}
template <int KIND, int TYPE>
static int product_group(ProductArgs& p) {
  switch (p.w.group) {
    case 32: return product_tiles<KIND, TYPE, 32>(p);
    case 64: return product_tiles<KIND, TYPE, 64>(p);
    default: return product_tiles<KIND, TYPE, 128>(p);
  }
}
template <int TYPE>
static int product_kind(ProductArgs& p) {
  switch (p.a.kind) {
    case HERSCHEL_FP8: return product_group<HERSCHEL_FP8, TYPE>(p);
    case HERSCHEL_INT8: return product_group<HERSCHEL_INT8, TYPE>(p);
    default: return product_group<TYPE, TYPE>(p);
  }
}

}  // namespace hop

extern "C" int herschel_product4(const herschel_product_args* args, const herschel_weights4* weights) {
  using namespace hop;
  if (!args || !weights) return HERSCHEL_EINVAL;
  const herschel_product_args& a = *args;
  const herschel_weights4& w = *weights;
  if (w.n < 1 || w.k < 1 || (w.group != 32 && w.group != 64 && w.group != 128) || !type_ok(w.scale_type))
    return HERSCHEL_EINVAL;
  if (w.k > 0x7fffff00 || w.n > 0x7ffffff0) return HERSCHEL_EINVAL;  // filled up they stay in 31 bits
  if (!w.codes || !w.scales || !aligned(w.codes, 16) || !aligned(w.scales, 16) || !aligned(w.zeros, 16))
    return HERSCHEL_EINVAL;
  if (!type_ok(a.type) || (a.kind != a.type && !quantised(a.kind)) || a.n_rows < 0 || a.x_row < 0) return HERSCHEL_EINVAL;
  if (a.x_group && (!quantised(a.kind) || a.x_group != w.group)) return HERSCHEL_EINVAL;
  if (a.gated && w.n % 32) return HERSCHEL_EINVAL;
  if (a.n_rows == 0) return HERSCHEL_OK;  // nothing to point at
  if (!a.x || !a.out || !aligned(a.out, 2) || !aligned(a.x, quantised(a.kind) ? 1 : 2)) return HERSCHEL_EINVAL;
  if (quantised(a.kind) && (!a.x_scale || !aligned(a.x_scale, 4))) return HERSCHEL_EINVAL;
  ProductArgs p{a, w, (w.k + 127) / 128, w.n / 32};
  return a.type == HERSCHEL_BF16 ? product_kind<HERSCHEL_BF16>(p) : product_kind<HERSCHEL_F16>(p);
}
