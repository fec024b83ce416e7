// Rotary positions and the quantising write into the paged cache, one launch.
//
// A row (one head of one token) is read once, rotated in 32 bits, written
// rotated and, for keys and values, encoded into its cache row: the traffic is
// the floor, each input read and each output written once, plus the tables'
// rows.  The kernel is bound by that traffic: 8192 tokens of 32 query and 8 key
// heads of 128 into an fp8 cache, 206 MB, 34.5 us, 6.0 TB/s.  A decode step's 32
// tokens take 4.2 us, a launch's latency.
#include "ops.hpp"

namespace hop {

struct RopeArgs {
  herschel_rope_args a;
  herschel_cache c;  // k == nullptr: no cache
  int page_shift;
  int groups;        // vector form: row groups of a workgroup that share a token
  int parts;         // vector form: workgroups that share a token
};

// The codes' scale of a row whose largest magnitude has these bits, and its
// inverse; NaN and 0 if the row holds an infinity or a NaN.
template <int KIND>
__device__ __forceinline__ float row_scale(uint32_t amax_bits, float& inv) {
  if (amax_bits >= 0x7f800000u) {
    inv = 0.0f;
    return __builtin_nanf("");
  }
  const float s = fmaxf(__builtin_bit_cast(float, amax_bits) * (1.0f / code_max(KIND)), SCALE_MIN);
  inv = 1.0f / s;
  return s;
}
template <int KIND>
__device__ __forceinline__ uint32_t encode4(const float* x, float inv) {
  constexpr float M = code_max(KIND);
  float y[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    // 0 * NaN in a row without a scale: the code is 0 there
    const float z = inv == 0.0f ? 0.0f : x[i] * inv;
    y[i] = __builtin_amdgcn_fmed3f(z, -M, M);
  }
  if constexpr (KIND == HERSCHEL_FP8) {
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], w, true);
  } else {
    uint32_t w = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) w |= ((uint32_t)(int)__builtin_rintf(y[i]) & 0xffu) << (8 * i);
    return w;
  }
}

// Rotates pairs (a[i], b[i]); contraction off: each product and sum is rounded,
// so that the codes do not depend on which of them a compiler fuses.
__device__ __forceinline__ void rotate(float& a, float& b, float c, float s) {
#pragma clang fp contract(off)
  const float p = a * c, q = b * s, r = b * c, t = a * s;
  a = p - q;
  b = r + t;
}

// Vector form.  A group of G lanes (G = head_dim / 16 rounded up to a power of
// two) holds a row, 16 elements a lane in two chunks of 16 bytes: both
// elements of every pair in one lane, and the row's maximum a few lane
// exchanges away.  A group takes several rows of one token, so the token's cos
// and sin are read once for them.  KIND -1: no cache.
template <int TYPE, int KIND, int LAYOUT, int G>
__global__ __launch_bounds__(256) void k_rope(RopeArgs p) {
  const herschel_rope_args& a = p.a;
  const int lane = threadIdx.x % G, group = threadIdx.x / G;
  const int D = a.head_dim, R = a.rotary_dim;
  const int sub = group % p.groups + p.groups * (blockIdx.x % p.parts), step = p.groups * p.parts;
  const int64_t t = (int64_t)(blockIdx.x / p.parts) * (256 / G / p.groups) + group / p.groups;
  if (t >= a.n_tokens) return;
  const bool holds = lane * 16 < D, turns = lane * 16 < R;
  // where the lane's two chunks are: the two sides of eight pairs, or neighbours
  const int at0 = LAYOUT == HERSCHEL_ROPE_HALF && turns ? lane * 8 : lane * 16;
  const int at1 = LAYOUT == HERSCHEL_ROPE_HALF && turns ? lane * 8 + R / 2 : lane * 16 + 8;

  const int64_t pos = a.positions[t];
  const bool placed = pos >= 0 && pos < a.n_positions;
  float cs[8], sn[8];
  if (turns) {
    const f32x4* tab = (const f32x4*)(a.table + ((placed ? pos : 0) * (R / 2) + lane * 8) * 2);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const f32x4 x = tab[i];
      cs[2 * i] = placed ? x[0] : __builtin_nanf("");
      sn[2 * i] = x[1];
      cs[2 * i + 1] = placed ? x[2] : __builtin_nanf("");
      sn[2 * i + 1] = x[3];
    }
  }
  int64_t row0 = -1;  // the token's row of head 0 in the cache
  if constexpr (KIND >= 0) {
    const int64_t slot = a.slots[t], page = slot >> p.page_shift;
    if (slot >= 0 && page < p.c.n_pages && placed)
      row0 = ((page * p.c.n_heads) << p.page_shift) + (slot & (p.c.page_size - 1));
    if (sub == 0 && lane == 0 && slot >= 0 && page >= p.c.n_pages) flag(a.status, HERSCHEL_OP_BAD_SLOT);
  }
  if (sub == 0 && lane == 0 && !placed) flag(a.status, HERSCHEL_OP_BAD_POSITION);

  const int nq = a.q ? a.q_heads : 0, nk = a.k ? a.kv_heads : 0, nv = KIND >= 0 && a.k ? a.kv_heads : 0;
  for (int h = sub; h < nq + nk + nv; h += step) {
    const int part = h < nq ? 0 : h < nq + nk ? 1 : 2;  // query, key, value
    const int head = part == 0 ? h : part == 1 ? h - nq : h - nq - nk;
    const herschel_strides st = part == 0 ? a.q_strides : part == 1 ? a.k_strides : a.v_strides;
    const uint16_t* src = (const uint16_t*)(part == 0 ? a.q : part == 1 ? a.k : a.v) + t * st.row + head * st.head;
    u32x4 w0 = {0, 0, 0, 0}, w1 = {0, 0, 0, 0};
    if (holds) {
      w0 = *(const u32x4*)(src + at0);
      w1 = *(const u32x4*)(src + at1);
    }
    float x[16];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      unpack2<TYPE>(w0[i], x[2 * i], x[2 * i + 1]);
      unpack2<TYPE>(w1[i], x[8 + 2 * i], x[9 + 2 * i]);
    }
    if (turns && part < 2) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        if constexpr (LAYOUT == HERSCHEL_ROPE_HALF) rotate(x[i], x[i + 8], cs[i], sn[i]);
        else rotate(x[2 * i], x[2 * i + 1], cs[i], sn[i]);
      }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      w0[i] = pack2<TYPE>(x[2 * i], x[2 * i + 1]);
      w1[i] = pack2<TYPE>(x[8 + 2 * i], x[9 + 2 * i]);
    }
    uint16_t* dst = part == 0 ? (uint16_t*)a.q_out : part == 1 ? (uint16_t*)a.k_out : nullptr;
    if (dst && holds) {
      const herschel_strides so = part == 0 ? a.q_out_strides : a.k_out_strides;
      dst += t * so.row + head * so.head;
      // past the caches, which hold what is still to be read: 8192 tokens 47.8 to 38.3 us,
      // with the codes as well 35.1
      __builtin_nontemporal_store(w0, (u32x4*)(dst + at0));
      __builtin_nontemporal_store(w1, (u32x4*)(dst + at1));
    }
    if constexpr (KIND >= 0) {
      if (part == 0 || row0 < 0) continue;
      const int64_t row = row0 + ((int64_t)head << p.page_shift);
      if constexpr (!quantised(KIND)) {
        if (holds) {
          uint16_t* to = (uint16_t*)(part == 1 ? p.c.k : p.c.v) + row * D;
          *(u32x4*)(to + at0) = w0;
          *(u32x4*)(to + at1) = w1;
        }
      } else {
        // magnitudes as bits order like the numbers, with infinity and NaN above all
        uint32_t m = 0;
#pragma unroll
        for (int i = 0; i < 16; ++i) m = max(m, __builtin_bit_cast(uint32_t, x[i]) & 0x7fffffffu);
#pragma unroll
        for (int o = 1; o < G; o *= 2) m = max(m, (uint32_t)__shfl_xor((int)m, o));
        float inv;
        const float scale = row_scale<KIND>(m, inv);
        if (holds) {
          uint8_t* to = (uint8_t*)(part == 1 ? p.c.k : p.c.v) + row * D;
          __builtin_nontemporal_store(u32x2{encode4<KIND>(x, inv), encode4<KIND>(x + 4, inv)}, (u32x2*)(to + at0));
          __builtin_nontemporal_store(u32x2{encode4<KIND>(x + 8, inv), encode4<KIND>(x + 12, inv)}, (u32x2*)(to + at1));
          if (lane == 0) (part == 1 ? p.c.k_scale : p.c.v_scale)[row] = scale;
        }
      }
    }
  }
}

// Element form, for head sizes, rotary sizes, strides or addresses that the
// chunks above do not fit: a wave per row, one or two pairs a lane.
template <int TYPE, int KIND>
__global__ __launch_bounds__(256) void k_rope_elements(RopeArgs p) {
  const herschel_rope_args& a = p.a;
  const int D = a.head_dim, R = a.rotary_dim, lane = threadIdx.x % WAVE;
  const int nq = a.q ? a.q_heads : 0, nk = a.k ? a.kv_heads : 0, nv = KIND >= 0 && a.k ? a.kv_heads : 0;
  const int64_t r = (int64_t)blockIdx.x * (256 / WAVE) + threadIdx.x / WAVE, t = r / (nq + nk + nv);
  if (t >= a.n_tokens) return;
  const int h = (int)(r % (nq + nk + nv));
  const int part = h < nq ? 0 : h < nq + nk ? 1 : 2;
  const int head = part == 0 ? h : part == 1 ? h - nq : h - nq - nk;
  const herschel_strides st = part == 0 ? a.q_strides : part == 1 ? a.k_strides : a.v_strides;
  const uint16_t* src = (const uint16_t*)(part == 0 ? a.q : part == 1 ? a.k : a.v) + t * st.row + head * st.head;
  const int64_t pos = a.positions[t];
  const bool placed = pos >= 0 && pos < a.n_positions;
  int64_t row = -1;
  if constexpr (KIND >= 0) {
    const int64_t slot = a.slots[t], page = slot >> p.page_shift;
    if (slot >= 0 && page < p.c.n_pages && placed)
      row = ((page * p.c.n_heads + head) << p.page_shift) + (slot & (p.c.page_size - 1));
    if (h == 0 && lane == 0 && slot >= 0 && page >= p.c.n_pages) flag(a.status, HERSCHEL_OP_BAD_SLOT);
  }
  if (h == 0 && lane == 0 && !placed) flag(a.status, HERSCHEL_OP_BAD_POSITION);
  float x[2][2] = {{0, 0}, {0, 0}};
  int at[2][2];
  uint32_t m = 0;
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    const int i = lane + e * WAVE;  // pair
    const bool turns = i < R / 2;
    const bool half = a.layout == HERSCHEL_ROPE_HALF;
    at[e][0] = turns && half ? i : 2 * i;  // beyond the rotated part: neighbours
    at[e][1] = turns && half ? i + R / 2 : 2 * i + 1;
    if (i >= D / 2) continue;
    float unused;
    unpack2<TYPE>(src[at[e][0]], x[e][0], unused);
    unpack2<TYPE>(src[at[e][1]], x[e][1], unused);
    if (turns && part < 2) {
      const float* cs = a.table + ((placed ? pos : 0) * (R / 2) + i) * 2;
      rotate(x[e][0], x[e][1], placed ? cs[0] : __builtin_nanf(""), cs[1]);
    }
#pragma unroll
    for (int j = 0; j < 2; ++j) m = max(m, __builtin_bit_cast(uint32_t, x[e][j]) & 0x7fffffffu);
  }
  float inv = 0, scale = 0;
  if constexpr (KIND >= 0 && quantised(KIND)) {
#pragma unroll
    for (int o = 1; o < WAVE; o *= 2) m = max(m, (uint32_t)__shfl_xor((int)m, o));
    scale = row_scale<KIND>(m, inv);
  }
  uint16_t* dst = part == 0 ? (uint16_t*)a.q_out : part == 1 ? (uint16_t*)a.k_out : nullptr;
  const herschel_strides so = part == 0 ? a.q_out_strides : a.k_out_strides;
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    if (lane + e * WAVE >= D / 2) continue;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const uint16_t w = (uint16_t)pack2<TYPE>(x[e][j], 0.0f);
      if (dst) dst[t * so.row + head * so.head + at[e][j]] = w;
      if constexpr (KIND >= 0) {
        if (part == 0 || row < 0) continue;
        if constexpr (!quantised(KIND)) {
          ((uint16_t*)(part == 1 ? p.c.k : p.c.v))[row * D + at[e][j]] = w;
        } else {
          const float one[4] = {x[e][j], 0, 0, 0};
          ((uint8_t*)(part == 1 ? p.c.k : p.c.v))[row * D + at[e][j]] = (uint8_t)encode4<KIND>(one, inv);
          if (lane == 0 && e == 0 && j == 0) (part == 1 ? p.c.k_scale : p.c.v_scale)[row] = scale;
        }
      }
    }
  }
}

template <int TYPE, int KIND>
static int rope_launch(RopeArgs& p) {
  const herschel_rope_args& a = p.a;
  const int rows = (a.q ? a.q_heads : 0) + (a.k ? a.kv_heads * (KIND >= 0 ? 2 : 1) : 0);
  bool vec = a.head_dim % 16 == 0 && a.rotary_dim % 16 == 0 && aligned(a.table, 16);
  vec = vec && (!a.q || chunks_aligned(a.q, a.q_strides)) && (!a.q_out || chunks_aligned(a.q_out, a.q_out_strides));
  vec = vec && (!a.k || chunks_aligned(a.k, a.k_strides)) && (!a.k_out || chunks_aligned(a.k_out, a.k_out_strides));
  vec = vec && (KIND < 0 || !a.k || chunks_aligned(a.v, a.v_strides));
  if (!vec) {
    const int64_t blocks = (a.n_tokens * rows + 3) / 4;
    if (blocks > 0x7fffffff) return HERSCHEL_EINVAL;
    return launch(k_rope_elements<TYPE, KIND>, dim3((unsigned)blocks), dim3(256), 0, a.hip_stream, p);
  }
  // Lanes of a row, row groups that share a token, and workgroups that share
  // it.  Few tokens: as many groups as rows, one row each, the launch's time
  // is latency.  Many: a group takes up to three rows with one load of cos and sin.
  const int G = a.head_dim <= 64 ? 4 : a.head_dim <= 128 ? 8 : 16, per = 256 / G;
  const bool few = a.n_tokens * rows < 16384;
  p.groups = per;
  p.parts = 1;
  while (p.groups > 1 && p.groups / 2 * (few ? 1 : 3) >= rows) p.groups /= 2;
  if (p.groups == per) p.parts = (rows + per * (few ? 1 : 3) - 1) / (per * (few ? 1 : 3));
  const int tokens = per / p.groups;
  const int64_t blocks = (a.n_tokens + tokens - 1) / tokens * p.parts;
  if (blocks > 0x7fffffff) return HERSCHEL_EINVAL;
  const bool half = a.layout == HERSCHEL_ROPE_HALF;
  void (*k)(RopeArgs) =
      G == 4   ? (half ? k_rope<TYPE, KIND, HERSCHEL_ROPE_HALF, 4> : k_rope<TYPE, KIND, HERSCHEL_ROPE_INTERLEAVED, 4>)
      : G == 8 ? (half ? k_rope<TYPE, KIND, HERSCHEL_ROPE_HALF, 8> : k_rope<TYPE, KIND, HERSCHEL_ROPE_INTERLEAVED, 8>)
               : (half ? k_rope<TYPE, KIND, HERSCHEL_ROPE_HALF, 16> : k_rope<TYPE, KIND, HERSCHEL_ROPE_INTERLEAVED, 16>);
  return launch(k, dim3((unsigned)blocks), dim3(256), 0, a.hip_stream, p);
}

template <int TYPE>
static int rope_kind(RopeArgs& p, int kind) {
  switch (kind) {
    case -1: return rope_launch<TYPE, -1>(p);
    case HERSCHEL_FP8: return rope_launch<TYPE, HERSCHEL_FP8>(p);
    case HERSCHEL_INT8: return rope_launch<TYPE, HERSCHEL_INT8>(p);
    default: return rope_launch<TYPE, TYPE>(p);
  }
}

}  // namespace hop

extern "C" int herschel_rope_write(const herschel_rope_args* args, const herschel_cache* cache) {
  using namespace hop;
  if (!args) return HERSCHEL_EINVAL;
  const herschel_rope_args& a = *args;
  if (a.n_tokens < 0 || a.head_dim < 2 || a.head_dim > 256 || (a.head_dim & 1) || !type_ok(a.type)) return HERSCHEL_EINVAL;
  if (a.rotary_dim < 0 || a.rotary_dim > a.head_dim || (a.rotary_dim & 1)) return HERSCHEL_EINVAL;
  if (a.layout != HERSCHEL_ROPE_HALF && a.layout != HERSCHEL_ROPE_INTERLEAVED) return HERSCHEL_EINVAL;
  if (!strides_ok(a.q_strides) || !strides_ok(a.k_strides) || !strides_ok(a.v_strides) ||
      !strides_ok(a.q_out_strides) || !strides_ok(a.k_out_strides))
    return HERSCHEL_EINVAL;
  if (cache && (!cache_ok(cache) || cache->head_dim != a.head_dim || cache->n_heads != a.kv_heads ||
                (!quantised(cache->kind) && cache->kind != a.type)))
    return HERSCHEL_EINVAL;
  if (a.n_tokens == 0) return HERSCHEL_OK;  // nothing to point at
  if ((!a.q && !a.k) || (a.q && a.q_heads < 1) || (a.k && a.kv_heads < 1)) return HERSCHEL_EINVAL;
  if ((a.q_out && !a.q) || (a.k_out && !a.k) || (cache && (!a.k || !a.v || !a.slots))) return HERSCHEL_EINVAL;
  if ((a.q && a.q_heads > (1 << 16)) || (a.k && a.kv_heads > (1 << 16))) return HERSCHEL_EINVAL;
  if (!a.positions || a.n_positions < 1 || (a.rotary_dim && (!a.table || !aligned(a.table, 8)))) return HERSCHEL_EINVAL;
  RopeArgs p{};
  p.a = a;
  if (cache) {
    p.c = *cache;
    p.page_shift = log2i(cache->page_size);
  }
  const int kind = cache ? cache->kind : -1;
  return a.type == HERSCHEL_BF16 ? rope_kind<HERSCHEL_BF16>(p, kind) : rope_kind<HERSCHEL_F16>(p, kind);
}
