// Attention over packed prompts.
//
// 4 head_dim flops per visible (query, key) pair and head against a few bytes
// per row: bound by the matrix cores, if softmax and operand traffic keep up.
//
//  - Both products are computed transposed, S^T = K Q^T and O^T = V^T P^T, with
//    32 x 32 x 16 instructions: lane n (and n + 32) holds scores of query row n
//    only, so a row's maximum, sum and scaling factor are the lane's own, and the
//    scores leave the first product in the lanes where the second wants them if
//    it takes its keys in the order 8 a + 4 g + i (g = lane / 32).  P never moves.
//  - Keys lie in LDS by rows, values transposed, by dimensions, with each 16
//    keys in that order, so that every operand is one 16-byte LDS read. The
//    chunks of a row are permuted by the row's number (K) and by the dimension's
//    (V), which spreads the reads of a wave over all banks.
//  - The transposition happens between global memory and LDS: a thread loads 8
//    dimensions of 4 keys and rearranges them with byte permutes, once for the
//    four waves that use them.
//  - Tiles whose keys all rows see run without a mask; tiles that no row sees
//    are not visited.
#include "ops.hpp"

namespace hop {

constexpr int QROWS = 128;  // query rows of a workgroup, 32 a wave
constexpr int KT = 64;      // keys of a tile
constexpr float LAZY_BY = 8.0f;
constexpr float NO_KEY = -3.0e38f;

struct PromptArgs {
  herschel_prompt_args a;
  int group;
  int levels;  // query tiles of the longest sequence
};

template <int TYPE, int D, bool VEC>
__global__ __launch_bounds__(256, 2) void k_prompt(PromptArgs p) {
  const herschel_prompt_args& a = p.a;
  constexpr int NC = D / 8;    // 16-byte chunks of a K row
  constexpr int DT = D / 32;   // blocks of dimensions
  __shared__ __align__(16) char s_k[2][KT * D * 2];
  __shared__ __align__(16) char s_v[2][D * KT * 2];

  const int tid = threadIdx.x, lane = tid % WAVE, wave = tid / WAVE, n = lane % 32, g = lane / 32;
  // longest tiles first: those at the end of a causal sequence
  int64_t id = blockIdx.x;
  const int qh = (int)(id % a.q_heads);
  id /= a.q_heads;
  const int b = (int)(id % a.n_seqs), level = p.levels - 1 - (int)(id / a.n_seqs);
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
  const bool real = row < nq;
  const int to = !real ? 0 : a.causal ? min(nk, max(0, row + shift + 1)) : nk;
  const int from = a.window > 0 ? max(0, row + shift - a.window + 1) : 0;
  // the workgroup's
  const int last = min(row0 + QROWS, nq) - 1;
  const int wg_to = a.causal ? min(nk, max(0, last + shift + 1)) : nk;
  const int wg_from = a.window > 0 ? max(0, row0 + shift - a.window + 1) / KT * KT : 0;
  // what every row of this wave sees
  const int first_row = row0 + wave * 32, last_row = first_row + 31;
  const int all_to = last_row >= nq ? 0 : a.causal ? min(nk, max(0, first_row + shift + 1)) : nk;
  const int all_from = a.window > 0 ? max(0, last_row + shift - a.window + 1) : 0;

  u32x4 q[D / 16];
  {
    const uint16_t* src = (const uint16_t*)a.q + (q0 + min(row, nq - 1)) * a.q_strides.row + qh * a.q_strides.head;
#pragma unroll
    for (int s = 0; s < D / 16; ++s)
      q[s] = VEC ? *(const u32x4*)(src + 16 * s + 8 * g) : load_elements(src + 16 * s + 8 * g);
  }
  f32x16 o[DT];
#pragma unroll
  for (int d = 0; d < DT; ++d)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[d][i] = 0;
  float ref = NO_KEY, sum = 0;
  const float to_log2 = a.scale * 1.44269504088896340736f;

  // A thread's share of a tile: K chunks tid, tid + 256, ... by rows; of V eight
  // dimensions of four keys.  Rows past the sequence's end read its last row.
  constexpr int KL = KT * NC / 256;
  constexpr int VT = D / 8;               // threads across the dimensions
  const uint16_t* kbase = (const uint16_t*)a.k + kk0 * a.k_strides.row + kh * a.k_strides.head;
  const uint16_t* vbase = (const uint16_t*)a.v + kk0 * a.v_strides.row + kh * a.v_strides.head;
  const int vd = tid % VT, vq = tid / VT;  // dimension block, key quad
  u32x4 kreg[KL], vreg[4];
  auto load_tile = [&](int k0) {
#pragma unroll
    for (int i = 0; i < KL; ++i) {
      const int c = tid + i * 256, key = min(k0 + c / NC, nk - 1);
      const uint16_t* s = kbase + key * a.k_strides.row + c % NC * 8;
      kreg[i] = VEC ? *(const u32x4*)s : load_elements(s);
    }
    if (vq < KT / 4) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int key = min(k0 + vq * 4 + j, nk - 1);
        const uint16_t* s = vbase + key * a.v_strides.row + vd * 8;
        vreg[j] = VEC ? *(const u32x4*)s : load_elements(s);
      }
    }
  };
  auto store_tile = [&](int buf) {
#pragma unroll
    for (int i = 0; i < KL; ++i) {
      const int c = tid + i * 256, key = c / NC, ch = c % NC;
      *(u32x4*)(s_k[buf] + key * (D * 2) + ((ch ^ (key & (NC - 1))) * 16)) = kreg[i];
    }
    if (vq < KT / 4) {
      // four keys of dimension 8 vd + e as 8 bytes: keys 8 hi + 4 g + (0..3) of 16 go to half hi of chunk 2 s + g
      const int s16 = vq / 4, hi = vq / 2 % 2, gg = vq % 2;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const uint32_t sel = e & 1 ? 0x07060302u : 0x05040100u;
        const u32x2 w = {__builtin_amdgcn_perm(vreg[1][e / 2], vreg[0][e / 2], sel),
                         __builtin_amdgcn_perm(vreg[3][e / 2], vreg[2][e / 2], sel)};
        const int d = vd * 8 + e, ch = (2 * s16 + gg) ^ ((d ^ (d >> 3)) & 7);
        *(u32x2*)(s_v[buf] + d * (KT * 2) + ch * 16 + hi * 8) = w;
      }
    }
  };

  int buf = 0;
  if (wg_from < wg_to) {
    load_tile(wg_from);
    store_tile(0);
  }
  __syncthreads();
  for (int k0 = wg_from; k0 < wg_to; k0 += KT, buf ^= 1) {
    const bool more = k0 + KT < wg_to;
    if (more) load_tile(k0 + KT);
    // S^T: two blocks of 32 keys
    f32x16 sc[2];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
#pragma unroll
      for (int i = 0; i < 16; ++i) sc[t][i] = 0;
#pragma unroll
      for (int s = 0; s < D / 16; ++s) {
        const int key = 32 * t + n;
        const u32x4 ka = *(const u32x4*)(s_k[buf] + key * (D * 2) + (((2 * s + g) ^ (key & (NC - 1))) * 16));
        sc[t] = mfma32<TYPE>(ka, q[s], sc[t]);
      }
    }
    const bool edge = k0 + KT > all_to || k0 < all_from;
    float x[32];
#pragma unroll
    for (int i = 0; i < 32; ++i) x[i] = sc[i / 16][i % 16] * to_log2;
    uint32_t seen = ~0u;
    if (edge) {
#pragma unroll
      for (int i = 0; i < 32; ++i) {
        const int key = k0 + 32 * (i / 16) + 8 * (i % 16 / 4) + 4 * g + i % 4;
        if (!(key < to && key >= from)) {
          x[i] = -INFINITY;
          seen &= ~(1u << i);
        }
      }
    }
    float top = x[0];
#pragma unroll
    for (int i = 1; i < 32; ++i) top = fmaxf(top, x[i]);
    if (__ballot(top > ref + LAZY_BY)) {
      const float t = fmaxf(ref, fmaxf(top, __shfl_xor(top, 32))), by = __builtin_amdgcn_exp2f(ref - t);
      ref = t;
      sum *= by;
#pragma unroll
      for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[d][i] *= by;
    }
    u32x4 pb[4];
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const float e0 = __builtin_amdgcn_exp2f(x[2 * i] - ref), e1 = __builtin_amdgcn_exp2f(x[2 * i + 1] - ref);
      sum += e0 + e1;
      pb[i / 4][i % 4] = pack2<TYPE>(e0, e1);
    }
    // O^T += V^T P^T
#pragma unroll
    for (int d = 0; d < DT; ++d) {
#pragma unroll
      for (int s = 0; s < 4; ++s) {
        const int dim = 32 * d + n;
        const u32x4 va =
            *(const u32x4*)(s_v[buf] + dim * (KT * 2) + (((2 * s + g) ^ ((dim ^ (dim >> 3)) & 7)) * 16));
        if (!edge) {
          o[d] = mfma32<TYPE>(va, pb[s], o[d]);
        } else {
          // a value that is not finite reaches the rows that see its key and no
          // other: it is taken out of the product and added where seen
          constexpr uint32_t ONE = TYPE == HERSCHEL_BF16 ? 0x3f80u : 0x3c00u;
          constexpr uint32_t INF = TYPE == HERSCHEL_BF16 ? 0x7f80u : 0x7c00u;
          u32x4 bad, ok;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            bad[i] = not_finite2<TYPE>(va[i]);
            ok[i] = va[i] & ~bad[i];
          }
          o[d] = mfma32<TYPE>(ok, pb[s], o[d]);
          if (__ballot((bad[0] | bad[1] | bad[2] | bad[3]) != 0)) {
            u32x4 up, down, sees;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const uint32_t two = seen >> (8 * s + 2 * i);
              sees[i] = (two & 1 ? ONE : 0u) | (two & 2 ? ONE << 16 : 0u);
              uint32_t u = 0, dn = 0;
#pragma unroll
              for (int h = 0; h < 32; h += 16) {
                const uint32_t z = (va[i] >> h) & 0xffffu;
                if ((bad[i] >> h) & 1) {
                  if (z != (INF | 0x8000u)) u |= ONE << h;
                  if (z != INF) dn |= ONE << h;
                }
              }
              up[i] = u;
              down[i] = dn;
            }
            f32x16 nu, nd;
#pragma unroll
            for (int i = 0; i < 16; ++i) nu[i] = nd[i] = 0;
            nu = mfma32<TYPE>(up, sees, nu);
            nd = mfma32<TYPE>(down, sees, nd);
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              if (nu[i] > 0) o[d][i] += INFINITY;
              if (nd[i] > 0) o[d][i] -= INFINITY;
            }
          }
        }
      }
    }
    if (more) store_tile(buf ^ 1);
    __syncthreads();
  }

  sum += __shfl_xor(sum, 32);
  if (!real) return;
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
  const int64_t blocks = (int64_t)p.levels * p.a.n_seqs * p.a.q_heads;
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
  PromptArgs p{a, a.q_heads / a.kv_heads, (a.max_q + QROWS - 1) / QROWS};
  const bool vec = chunks_aligned(a.q, a.q_strides) && chunks_aligned(a.k, a.k_strides) && chunks_aligned(a.v, a.v_strides);
  const bool bf = a.type == HERSCHEL_BF16;
  if (a.head_dim == 64) return bf ? prompt_launch<HERSCHEL_BF16, 64>(p, vec) : prompt_launch<HERSCHEL_F16, 64>(p, vec);
  return bf ? prompt_launch<HERSCHEL_BF16, 128>(p, vec) : prompt_launch<HERSCHEL_F16, 128>(p, vec);
}
