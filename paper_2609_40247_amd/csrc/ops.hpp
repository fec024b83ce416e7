// Shared pieces of the reference operators (rotary write, cache read, prompt
// and decode attention): element types, conversions, the cache's addressing
// and the host's launch helper.  Sums, maxima and scales are 32-bit floats;
// elements are bf16 or half, cache codes 8 bits.
#pragma once

#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "herschel_ops.h"

namespace hop {

constexpr int WAVE = 64;

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

// Codes' largest magnitude.
__host__ __device__ constexpr float code_max(int kind) { return kind == HERSCHEL_FP8 ? 448.0f : 127.0f; }
// The smallest scale of a row: 1 / scale stays finite, and rows of zeros need no case of their own.
constexpr float SCALE_MIN = 0x1p-100f;

__host__ __device__ constexpr bool quantised(int kind) { return kind == HERSCHEL_FP8 || kind == HERSCHEL_INT8; }
__host__ __device__ constexpr int code_bytes(int kind) { return quantised(kind) ? 1 : 2; }

// Two floats rounded to nearest even into a word of TYPE, the first in the low half, and back.
template <int TYPE>
__device__ __forceinline__ uint32_t pack2(float a, float b) {
  const f32x2 x = {a, b};
  if constexpr (TYPE == HERSCHEL_BF16) return __builtin_bit_cast(uint32_t, __builtin_convertvector(x, bf16x2));
  else return __builtin_bit_cast(uint32_t, __builtin_convertvector(x, f16x2));
}
template <int TYPE>
__device__ __forceinline__ void unpack2(uint32_t w, float& a, float& b) {
  if constexpr (TYPE == HERSCHEL_BF16) {
    a = __builtin_bit_cast(float, w << 16);
    b = __builtin_bit_cast(float, w & 0xffff0000u);
  } else {
    const f16x2 h = __builtin_bit_cast(f16x2, w);
    a = (float)h[0];
    b = (float)h[1];
  }
}
// Bytes 2 HI and 2 HI + 1 of a word of codes as two elements of TYPE: both
// kinds of code are exact in either type (at most 8 significant bits, fp8's
// smallest step 2^-9 is a normal half).
template <int KIND, int TYPE, bool HI>
__device__ __forceinline__ uint32_t decode2(uint32_t w) {
  if constexpr (KIND == HERSCHEL_FP8) {
    if constexpr (TYPE == HERSCHEL_BF16)
      return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, HI));
    else
      return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.0f, HI));
  } else {
    const int x = (int)w;
    return pack2<TYPE>((float)(int)(int8_t)(x >> (HI ? 16 : 0)), (float)(int)(int8_t)(x >> (HI ? 24 : 8)));
  }
}
// The same as floats.
template <int KIND, bool HI>
__device__ __forceinline__ void decode2f(uint32_t w, float& a, float& b) {
  if constexpr (KIND == HERSCHEL_FP8) {
    const auto f = __builtin_amdgcn_cvt_pk_f32_fp8(w, HI);
    a = f[0];
    b = f[1];
  } else {
    const int x = (int)w;
    a = (float)(int)(int8_t)(x >> (HI ? 16 : 0));
    b = (float)(int)(int8_t)(x >> (HI ? 24 : 8));
  }
}

// D += A B on the matrix cores: A[m][k] in lane m + M (k / 8), B[k][n] in lane
// n + M (k / 8), both element k % 8 of the lane's eight.
template <int TYPE>
__device__ __forceinline__ f32x4 mfma16(u32x4 a, u32x4 b, f32x4 c) {
  if constexpr (TYPE == HERSCHEL_BF16)
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0,
                                                   0, 0);
  else
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0,
                                                  0);
}
template <int TYPE>
__device__ __forceinline__ f32x16 mfma32(u32x4 a, u32x4 b, f32x16 c) {
  if constexpr (TYPE == HERSCHEL_BF16)
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0,
                                                   0, 0);
  else
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0,
                                                  0);
}

// Halves of a word of TYPE that hold an infinity or a NaN: 0xffff in their place.
template <int TYPE>
__device__ __forceinline__ uint32_t not_finite2(uint32_t w) {
  constexpr uint32_t E = TYPE == HERSCHEL_BF16 ? 0x7f80u : 0x7c00u;
  return ((w & E) == E ? 0xffffu : 0u) | (((w >> 16) & E) == E ? 0xffff0000u : 0u);
}

// The first key that a window of w keys up to key x holds (w 0: no window); for any w, as x - w may pass 32 bits.
__device__ __forceinline__ int window_from(int x, int w) { return w > 0 && x >= w ? x - w + 1 : 0; }

__device__ __forceinline__ void flag(uint32_t* status, uint32_t bit) {
  if (status) atomicOr(status, bit);
}

// The exponentials of a row are taken against a reference that stays while their
// sums show that it fits.  The second product takes them in TYPE, its sums and the
// exponentials' own are 32-bit.  That rounding is a choice: the product runs at the
// 16-bit rate, and a weight is off by half a last place of what the values
// themselves are given in (4096 rows of 32 heads in bf16 0.0021 from 64 bits where
// exponentials of 32 bits give 0.0016, most of it the output's own rounding).
//
// bf16 has the exponents of 32 bits: the largest that called for a move stands at
// 2^-30, so that sums of the largest values over a million keys stay numbers.  A half has 2^-24 to 65504: weights far below the largest
// would be lost from the product and stay in the sum, and where the largest has a
// value of 0, they are all there is.  So a move puts the largest at 2^6, and the
// reference moves down too, where a step's sum in a row is below 2^-12: what a key
// loses is at most 2^-25, 2^-31 of the row's largest, and with the 32 keys of a
// lane 2^-8 of what the step has.  Moves cost a step's exponentials twice, and
// rows whose scores spread over 20 powers of two move often: with a tenth of the
// heads so, prompts in half take 4 to 14% longer (4096 rows of 32 heads of 128 164
// us against 148), without such heads under 1%.
template <int TYPE>
struct Reference {
  static constexpr bool HALF = TYPE == HERSCHEL_F16;
  static constexpr float TOP = HALF ? 6.0f : -30.0f;           // a move up puts the largest at 2^TOP
  static constexpr float LARGE = HALF ? 65504.0f : 0x1p-18f;  // a lane's sum above this moves it up
  static constexpr float SMALL = 0x1p-12f;                    // below this, in all of a row's lanes, down
  static constexpr float LOW = -4.0f;                         // a move down puts the largest at 2^LOW
  // A step's sums s, PARTS lanes (64 / PARTS apart) to a row: whether the reference may have to move.
  template <int PARTS>
  static __device__ __forceinline__ bool off(float s) {
    if constexpr (!HALF) return __ballot(!(s <= LARGE)) != 0;
    constexpr uint32_t FROM = __builtin_bit_cast(uint32_t, SMALL), TO = __builtin_bit_cast(uint32_t, LARGE);
    if (__ballot(__builtin_bit_cast(uint32_t, s) - FROM > TO - FROM) == 0) return false;  // most steps; NaN is above
    uint64_t low = __ballot(s < SMALL), some = __ballot(s > 0.0f);
#pragma unroll
    for (int o = 32; o >= WAVE / PARTS; o /= 2) low &= low >> o, some |= some >> o;
    return (__ballot(!(s <= LARGE)) | (low & some & (~0ull >> (WAVE - WAVE / PARTS)))) != 0;
  }
  // The reference after a step whose largest score (a power of two) is top, for a row whose sum so far is
  // total.  Down by no more than leaves that sum below 2^60: what lies 2^60 below it is nothing.
  static __device__ __forceinline__ float moved(float ref, float top, float total) {
    if (HALF && top < ref - 11.0f && top > -3.0e38f)
      return fmaxf(top - LOW, ref + __builtin_amdgcn_logf(total) - 60.0f);
    return fmaxf(ref, top - TOP);
  }
};

// x times a weight that may be too small for 32 bits: 0 then, but an infinity or a NaN stays one.
__device__ __forceinline__ float weighted(float x, float by) { return by != 0 ? x * by : x - x == 0 ? 0.0f : x; }

// Natural log of sum times 2 to the ref.
__device__ __forceinline__ float log_sum(float ref, float sum) {
  if (sum == 0) return -INFINITY;
  return (ref + (float)__builtin_amdgcn_frexp_expf(sum) + __builtin_amdgcn_logf(__builtin_amdgcn_frexp_mantf(sum))) *
         0.69314718055994530942f;
}

// 16 bytes that may lie at any element (2 bytes).
__device__ __forceinline__ u32x4 load_elements(const uint16_t* p) {
  u32x4 r;
#pragma unroll
  for (int i = 0; i < 4; ++i) r[i] = (uint32_t)p[2 * i] | ((uint32_t)p[2 * i + 1] << 16);
  return r;
}

// ------------------------------------------------------------ host
// Launches and returns a HERSCHEL_* code; a failed launch leaves no error
// behind for the caller's next HIP call.
template <class Args>
inline int launch(void (*kernel)(Args), dim3 grid, dim3 block, size_t lds, void* stream, const Args& args) {
  Args copy = args;
  void* list[] = {&copy};
  if (hipLaunchKernel((const void*)kernel, grid, block, list, lds, (hipStream_t)stream) == hipSuccess)
    return HERSCHEL_OK;
  (void)hipGetLastError();
  return HERSCHEL_EDEVICE;
}

inline bool aligned(const void* p, size_t to) { return ((uintptr_t)p & (to - 1)) == 0; }
inline bool type_ok(int t) { return t == HERSCHEL_BF16 || t == HERSCHEL_F16; }
inline bool strides_ok(const herschel_strides& s) { return s.row >= 0 && s.head >= 0; }
// Every 16-byte chunk of the rows lies at a multiple of 16 bytes.
inline bool chunks_aligned(const void* p, const herschel_strides& s) {
  return aligned(p, 16) && (s.row & 7) == 0 && (s.head & 7) == 0;
}

inline bool cache_ok(const herschel_cache* c) {
  if (!c || !c->k || !c->v || c->n_pages < 1 || c->n_heads < 1 || c->kind < HERSCHEL_BF16 || c->kind > HERSCHEL_INT8)
    return false;
  const int p = c->page_size;
  if (p < 16 || p > 256 || (p & (p - 1)) || c->head_dim < 2 || c->head_dim > 256 || (c->head_dim & 1)) return false;
  if (!aligned(c->k, 16) || !aligned(c->v, 16)) return false;
  if (quantised(c->kind) && (!c->k_scale || !c->v_scale || !aligned(c->k_scale, 16) || !aligned(c->v_scale, 16)))
    return false;
  // rows are counted in 64 bits and a page's bytes in 31
  return c->n_pages < (1ll << 40) / ((int64_t)c->n_heads * p) &&
         (int64_t)c->n_heads * p * c->head_dim * code_bytes(c->kind) < (1ll << 31);
}
inline int log2i(int x) { return 31 - __builtin_clz((unsigned)x); }

}  // namespace hop
