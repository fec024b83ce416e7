// Attention over packed prompts.
//
// 4 head_dim flops per visible (query, key) pair and head against a few bytes
// per row: bound by the matrix cores, if softmax and operand traffic keep up.
//
//  - Both products are computed transposed, S^T = K Q^T and O^T = V^T P^T, with
//    32 x 32 x 16 instructions: lane n (and n + 32) holds scores of query row n
//    only, so a row's sum and scaling factor are the lane's own, and the scores
//    leave the first product in the lanes where the second wants them if it takes
//    its keys in the order 8 a + 4 g + i (g = lane / 32).  P never moves.
//  - A wave has 32 rows and two waves share a SIMD, of different workgroups: one
//    wave alone issues a VALU instruction every 6 cycles, two every 3, and the
//    exponentials of one run beside the products of the other.
//  - Keys lie in LDS by rows, copied there without passing registers; values
//    transposed, by dimensions, with each 16 keys in the order above, so that
//    every operand is one 16-byte read.  The chunks of a row are permuted by the
//    row's number (K) and by the dimension's (V), which spreads a wave's reads
//    over all banks.  The transposition is a thread's own: it loads 8 dimensions
//    of 4 keys and rearranges them with byte permutes.
//  - The reference of a row's exponentials stays as long as a tile's sum shows
//    that no exponential is large; then the maximum is taken and the
//    accumulators scaled.  No maximum is computed otherwise.
//  - Only tiles in which some row does not see some key are masked.  A hidden
//    key's exponential is 0, which an infinite or NaN value would turn into NaN:
//    in the tiles that may be masked such values go into LDS as 0, and if there
//    were any, they are added at the end to the rows that see them.
#include "ops.hpp"

namespace hop {

constexpr int QROWS = 128;  // query rows of a workgroup, 32 a wave
constexpr int KT = 64;      // keys of a tile
constexpr float NO_KEY = -3.0e38f;
constexpr float LARGE = 4096.0f;  // a sum above this moves the reference (half's largest value is 65504)

#define INLINE __attribute__((always_inline))

struct PromptArgs {
  herschel_prompt_args a;
  int group;
  int levels;  // query tiles of the longest sequence
  int spread;  // XCDs that share a key head's workgroups; 0: heads in turn
};

// A wave's copy of 64 chunks of 16 bytes from global memory to consecutive LDS.
__device__ __forceinline__ void copy_to_lds(const void* from, void* to) {
  __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)from,
                                   (__attribute__((address_space(3))) void*)to, 16, 0, 0);
}

template <int TYPE, int D, bool VEC>
__global__ __launch_bounds__(256, 2) void k_prompt(PromptArgs p) {
  const herschel_prompt_args& a = p.a;
  constexpr int NC = D / 8;    // 16-byte chunks of a K row
  constexpr int DT = D / 32;   // blocks of dimensions
  constexpr int NS = D / 16;   // steps of the first product
  constexpr int KBYTES = KT * D * 2;
  __shared__ __align__(16) char s_k[2 * KBYTES];
  __shared__ __align__(16) char s_v[2 * KBYTES];
  __shared__ int s_odd;  // values that are not finite in tiles that may be masked

  const int tid = threadIdx.x, lane = tid % WAVE, wave = __builtin_amdgcn_readfirstlane(tid / WAVE), n = lane % 32, g = lane / 32;
  // Longest tiles first (the end of a causal sequence); the heads of a key head
  // on one XCD, or on as few as there are, whose L2 then holds its keys.
  uint32_t id = blockIdx.x;
  int qh;
  if (p.spread) {
    const uint32_t xcd = id % 8;
    id = id / 8;
    const uint32_t heads = a.kv_heads > 8 ? (uint32_t)a.kv_heads / 8 : 1u;  // key heads of an XCD
    id = id * p.spread + xcd % p.spread;
    const uint32_t of = heads * p.group, h = id % of;  // query heads of an XCD, of one key head after the other
    qh = (int)(xcd / p.spread * of + h);
    id /= of;
  } else {
    qh = (int)(id % a.q_heads);
    id /= a.q_heads;
  }
  const int b = (int)(id % a.n_seqs), level = p.levels - 1 - (int)(id / a.n_seqs);
  if (level < 0) return;
  // lengths taken as the nearest valid
  const int64_t q0w = a.cu_q[b], q1w = a.cu_q[b + 1], k0w = a.cu_k[b], k1w = a.cu_k[b + 1];
  const int64_t q0 = min(max(q0w, (int64_t)0), a.n_q), q1 = min(max(q1w, q0), a.n_q);
  const int64_t kk0 = min(max(k0w, (int64_t)0), a.n_k), kk1 = min(max(k1w, kk0), a.n_k);
  const int nq = (int)min(q1 - q0, (int64_t)a.max_q), nk = (int)(kk1 - kk0);
  if (level == 0 && qh == 0 && tid == 0 && (q0 != q0w || q1 != q1w || kk0 != k0w || kk1 != k1w || q1 - q0 != nq))
    flag(a.status, HERSCHEL_OP_BAD_LENGTH);
  const int row0 = level * QROWS;
  if (row0 >= nq) return;
  const int kh = qh / p.group;
  const int shift = nk - (int)(q1 - q0);  // causal: row i sees keys up to i + shift

  // this lane's query row, and the keys it sees: [from, to)
  const int row = row0 + wave * 32 + n;
  const int to = row >= nq ? 0 : a.causal ? min(nk, max(0, row + shift + 1)) : nk;
  const int from = a.window > 0 ? max(0, row + shift - a.window + 1) : 0;
  // the workgroup's
  const int last = min(row0 + QROWS, nq) - 1;
  const int wg_to = a.causal ? min(nk, max(0, last + shift + 1)) : nk;
  const int wg_from = a.window > 0 ? min(wg_to, max(0, row0 + shift - a.window + 1)) / KT * KT : 0;
  const int tiles = (wg_to - wg_from + KT - 1) / KT;
  // keys outside these may be hidden from a row of this wave, of the workgroup
  const int first_row = row0 + wave * 32;
  const int all_to = first_row + 32 > nq ? 0 : a.causal ? min(nk, max(0, first_row + shift + 1)) : nk;
  const int all_from = a.window > 0 ? max(0, first_row + 31 + shift - a.window + 1) : 0;
  const int wg_all_to = row0 + QROWS > nq ? 0 : a.causal ? min(nk, max(0, row0 + shift + 1)) : nk;
  const int wg_all_from = a.window > 0 ? max(0, row0 + QROWS - 1 + shift - a.window + 1) : 0;

  // A negative scale goes into Q's signs: what is left is not negative.
  u32x4 q[NS];
  {
    const uint16_t* src = (const uint16_t*)a.q + (q0 + min(row, nq - 1)) * a.q_strides.row + qh * a.q_strides.head;
    const uint32_t sign = a.scale < 0 ? 0x80008000u : 0u;
#pragma unroll
    for (int s = 0; s < NS; ++s) {
      q[s] = VEC ? *(const u32x4*)(src + 16 * s + 8 * g) : load_elements(src + 16 * s + 8 * g);
      q[s] ^= sign;
    }
  }
  f32x16 o[DT];
#pragma unroll
  for (int d = 0; d < DT; ++d)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[d][i] = 0;
  float ref = NO_KEY, sum = 0;
  // not 0, so that a hidden key's minus infinity stays one: scores up to 2^80 then count as 0
  const float to_log2 = fmaxf(fabsf(a.scale) * 1.44269504088896340736f, 0x1p-100f);

  // A thread's share of a tile: chunks of K by rows; of V eight dimensions of
  // four keys.  Rows past the sequence's end read its last row.
  constexpr int KL = KT * NC / 256;
  constexpr int VT = D / 8;  // threads across the dimensions
  const uint16_t* kbase = (const uint16_t*)a.k + kk0 * a.k_strides.row + kh * a.k_strides.head;
  const uint16_t* vbase = (const uint16_t*)a.v + kk0 * a.v_strides.row + kh * a.v_strides.head;
  const int vd = tid % VT, vq = tid / VT;  // dimension block, key quad
  u32x4 vreg[4];
  // Whole tiles: one 32-bit offset a thread from addresses that are the
  // workgroup's.  LDS chunk c of a row holds the row's chunk c ^ row.
  const uint32_t koff = (uint32_t)((tid / NC) * a.k_strides.row + ((tid % NC) ^ (tid / NC & (NC - 1))) * 8) * 2;
  const uint32_t voff = (uint32_t)(vq * 4 * a.v_strides.row + vd * 8) * 2;
  auto load_k = [&](int tile, int buf) INLINE {
    const int k0 = wg_from + tile * KT;
    char* dst = s_k + buf * KBYTES + wave * WAVE * 16;
    if (VEC && k0 + KT <= nk) {
      const char* src = (const char*)(kbase + (int64_t)k0 * a.k_strides.row);
#pragma unroll
      for (int i = 0; i < KL; ++i) copy_to_lds(src + (int64_t)(i * (256 / NC)) * a.k_strides.row * 2 + koff, dst + i * 4096);
    } else {
      for (int i = 0; i < KL; ++i) {
        const int r = tid / NC + i * (256 / NC);
        const uint16_t* src = kbase + min(k0 + r, nk - 1) * a.k_strides.row + ((tid % NC) ^ (r & (NC - 1))) * 8;
        *(u32x4*)(dst + i * 4096 + lane * 16) = VEC ? *(const u32x4*)src : load_elements(src);
      }
    }
  };
  auto load_v = [&](int tile) INLINE {
    const int k0 = wg_from + tile * KT;
    if (D < 128 && vq >= KT / 4) return;
    if (VEC && k0 + KT <= nk) {
      const char* src = (const char*)(vbase + (int64_t)k0 * a.v_strides.row);
#pragma unroll
      for (int j = 0; j < 4; ++j) vreg[j] = *(const u32x4*)(src + (int64_t)j * a.v_strides.row * 2 + voff);
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const uint16_t* src = vbase + min(k0 + vq * 4 + j, nk - 1) * a.v_strides.row + vd * 8;
        vreg[j] = VEC ? *(const u32x4*)src : load_elements(src);
      }
    }
  };
  auto store_v = [&](int tile, int buf) INLINE {
    if (D >= 128 || vq < KT / 4) {
      const int k0 = wg_from + tile * KT;
      if (k0 + KT > wg_all_to || k0 < wg_all_from) {
        uint32_t any = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const uint32_t bad = not_finite2<TYPE>(vreg[j][i]);
            vreg[j][i] &= ~bad;
            any |= bad;
          }
        if (any) s_odd = 1;
      }
      // four keys of dimension 8 vd + e as 8 bytes: keys 8 hi + 4 g + (0..3) of 16 go to half hi of chunk 2 s + g
      const int s16 = vq / 4, hi = vq / 2 % 2, gg = vq % 2;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const uint32_t sel = e & 1 ? 0x07060302u : 0x05040100u;
        const u32x2 w = {__builtin_amdgcn_perm(vreg[1][e / 2], vreg[0][e / 2], sel),
                         __builtin_amdgcn_perm(vreg[3][e / 2], vreg[2][e / 2], sel)};
        const int d = vd * 8 + e, ch = (2 * s16 + gg) ^ ((d ^ (d >> 3)) & 7);
        *(u32x2*)(s_v + buf * KBYTES + d * (KT * 2) + ch * 16 + hi * 8) = w;
      }
    }
  };
  // operands: step s of the keys of half h of a tile; dimension block d, step s of the keys of half h
  auto read_k = [&](int buf, int h, int s) INLINE {
    const int key = 32 * h + n;
    return *(const u32x4*)(s_k + buf * KBYTES + key * (D * 2) + (((2 * s + g) ^ (key & (NC - 1))) * 16));
  };
  auto read_v = [&](int buf, int h, int d, int s) INLINE {
    const int dim = 32 * d + n;
    return *(const u32x4*)(s_v + buf * KBYTES + dim * (KT * 2) + (((4 * h + 2 * s + g) ^ ((dim ^ (dim >> 3)) & 7)) * 16));
  };
  f32x16 sc[2];
  u32x4 pb[4];
  // exponentials of the tile, rounded in pairs, and their sum
  auto exponentials = [&]() INLINE {
    float s = 0;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const float e0 = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[i / 8][2 * i % 16], to_log2, -ref));
      const float e1 = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[i / 8][2 * i % 16 + 1], to_log2, -ref));
      s += e0 + e1;
      pb[i / 4][i % 4] = pack2<TYPE>(e0, e1);
    }
    return s;
  };

  if (tid == 0) s_odd = 0;
  __syncthreads();
  if (tiles > 0) {
    load_k(0, 0);
    load_v(0);
    store_v(0, 0);
    __builtin_amdgcn_s_waitcnt(0);
    __syncthreads();
    for (int t = 0, buf = 0; t < tiles; ++t, buf ^= 1) {
      const bool more = t + 1 < tiles;
      if (more) {
        load_k(t + 1, buf ^ 1);
        load_v(t + 1);
      }
      const int k0 = wg_from + t * KT;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        f32x16 zero;
#pragma unroll
        for (int i = 0; i < 16; ++i) zero[i] = 0;
        sc[h] = mfma32<TYPE>(read_k(buf, h, 0), q[0], zero);
#pragma unroll
        for (int s = 1; s < NS; ++s) sc[h] = mfma32<TYPE>(read_k(buf, h, s), q[s], sc[h]);
      }
      if (k0 + KT > all_to || k0 < all_from) {
        const int lo = from - k0 - 4 * g, hi = to - k0 - 4 * g;
#pragma unroll
        for (int i = 0; i < 32; ++i) {
          const int c = 32 * (i / 16) + 8 * (i % 16 / 4) + i % 4;
          sc[i / 16][i % 16] = c < hi && c >= lo ? sc[i / 16][i % 16] : -INFINITY;
        }
      }
      float s = exponentials();
      if (__ballot(!(s <= LARGE))) {
        float top = sc[0][0];
#pragma unroll
        for (int i = 1; i < 32; ++i) top = fmaxf(top, sc[i / 16][i % 16]);
        top = fmaxf(top, __shfl_xor(top, 32));
        const float next = fmaxf(ref, top * to_log2), by = __builtin_amdgcn_exp2f(ref - next);
        ref = next;
        sum *= by;
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
          for (int i = 0; i < 16; ++i) o[d][i] *= by;
        s = exponentials();
      }
      sum += s;
#pragma unroll
      for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int k = 0; k < 4; ++k) o[d] = mfma32<TYPE>(read_v(buf, k / 2, d, k % 2), pb[k], o[d]);
      if (more) store_v(t + 1, buf ^ 1);
      __builtin_amdgcn_s_waitcnt(0);
      __syncthreads();
    }
    if (s_odd) {
      for (int key = wg_from; key < wg_to; ++key) {
        const int k0 = key / KT * KT;
        if (k0 + KT <= wg_all_to && k0 >= wg_all_from) continue;  // went through the product as they are
        const uint16_t* src = vbase + key * a.v_strides.row;
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const uint16_t w = src[32 * d + 8 * (i / 4) + 4 * g + i % 4];
            if (not_finite2<TYPE>(w) & 0xffffu) {
              float x, unused;
              unpack2<TYPE>(w, x, unused);
              if (key < to && key >= from) o[d][i] += x;
            }
          }
      }
    }
  }

  sum += __shfl_xor(sum, 32);
  if (row >= nq) return;
  const float inv = sum > 0 ? 1.0f / sum : sum == 0 ? 0.0f : sum;  // no key seen: 0; NaN stays
  const int64_t at = (q0 + row) * a.q_heads + qh;
#pragma unroll
  for (int d = 0; d < DT; ++d)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      uint16_t* out = (uint16_t*)a.out + at * D + 32 * d + 8 * i + 4 * g;
      *(u32x2*)out = u32x2{pack2<TYPE>(o[d][4 * i] * inv, o[d][4 * i + 1] * inv),
                           pack2<TYPE>(o[d][4 * i + 2] * inv, o[d][4 * i + 3] * inv)};
    }
  if (a.lse && g == 0) a.lse[at] = sum == 0 ? -INFINITY : (ref + __builtin_amdgcn_logf(sum)) * 0.69314718055994530942f;
}

template <int TYPE, int D>
static int prompt_launch(PromptArgs& p, bool vec) {
  // XCDs that share a key head: only where key heads and XCDs divide evenly
  const int G = p.a.kv_heads;
  p.spread = G >= 8 ? (G % 8 == 0 ? 1 : 0) : (8 % G == 0 ? 8 / G : 0);
  int64_t blocks = (int64_t)p.levels * p.a.n_seqs * p.a.q_heads;
  if (p.spread) blocks = (blocks / (G < 8 ? G : 8) + p.spread - 1) / p.spread * 8;
  if (blocks > 0x7fffffff) return HERSCHEL_EINVAL;
  return launch(vec ? k_prompt<TYPE, D, true> : k_prompt<TYPE, D, false>, dim3((unsigned)blocks), dim3(256), 0,
                p.a.hip_stream, p);
}

}  // namespace hop

extern "C" int herschel_attn_prompt(const herschel_prompt_args* args) {
  using namespace hop;
  if (!args) return HERSCHEL_EINVAL;
  const herschel_prompt_args& a = *args;
  if (a.n_seqs < 1 || a.n_q < 0 || a.n_k < 0 || a.max_q < 0 || a.n_q > 0x7fffffff || a.n_k > 0x7fffffff) return HERSCHEL_EINVAL;
  if (a.head_dim != 64 && a.head_dim != 128) return HERSCHEL_EINVAL;
  if (a.kv_heads < 1 || a.q_heads < 1 || a.q_heads % a.kv_heads || !type_ok(a.type)) return HERSCHEL_EINVAL;
  if (a.window < 0 || !isfinite(a.scale) || !a.cu_q || !a.cu_k) return HERSCHEL_EINVAL;
  if (!strides_ok(a.q_strides) || !strides_ok(a.k_strides) || !strides_ok(a.v_strides)) return HERSCHEL_EINVAL;
  if ((a.n_q && (!a.q || !a.out || !aligned(a.q, 2) || !aligned(a.out, 8))) ||
      (a.n_k && (!a.k || !a.v || !aligned(a.k, 2) || !aligned(a.v, 2))))
    return HERSCHEL_EINVAL;
  if (a.n_q == 0 || a.max_q == 0) return HERSCHEL_OK;
  PromptArgs p{a, a.q_heads / a.kv_heads, (a.max_q + QROWS - 1) / QROWS, 0};
  // 16-byte loads, and a tile's rows within 31 bits of bytes
  const bool vec = a.k_strides.row < (1 << 23) && a.v_strides.row < (1 << 23) && chunks_aligned(a.q, a.q_strides) && chunks_aligned(a.k, a.k_strides) && chunks_aligned(a.v, a.v_strides);
  const bool bf = a.type == HERSCHEL_BF16;
  if (a.head_dim == 64) return bf ? prompt_launch<HERSCHEL_BF16, 64>(p, vec) : prompt_launch<HERSCHEL_F16, 64>(p, vec);
  return bf ? prompt_launch<HERSCHEL_BF16, 128>(p, vec) : prompt_launch<HERSCHEL_F16, 128>(p, vec);
}
