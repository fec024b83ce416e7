// Attention of one or a few new tokens over the paged cache.
//
// Every visible key and value row is read once: 2 head_dim codes (and two
// scales) for 4 head_dim flops per query head, far below what the matrix cores
// need, so the kernel is bound by the reads.  Its shape follows from that:
//
//  - The rows that share a key head (its group of query heads times the new
//    tokens) are the columns of one matrix product, so each key is read once
//    for all of them.  The products are computed transposed, S^T = K Q^T and
//    O^T = V^T P^T: the score of (key 16 t + 4 g + i, row r) is then element i
//    of lane r + 16 g, and is in the place where the second product wants it if
//    that product takes its 32 keys in the order 4 g + i of the first sixteen,
//    then of the second.  A row's maximum and sum stay within a lane until the
//    end, and nothing goes through LDS.
//  - Keys and values go from the cache to registers in 16-byte chunks (8 for
//    8-bit values) whose lanes cover whole rows.  V^T needs eight keys of one
//    dimension in a lane: a lane loads eight dimensions of its eight keys, and a
//    byte permute per pair of elements transposes the 8 x 8 block.
//  - The work is cut by its length, not by sequence: all 128-key tiles of all
//    sequences and heads are laid end to end, and each workgroup takes an equal
//    share of the line, found from the lengths on the device.  Where a share ends
//    inside a sequence's head the parts are joined by a second small kernel.
//
// The reference of a row's exponentials is its maximum when last looked at: a
// score may exceed it by 2^8 before the accumulators are scaled anew, which is
// exact up to rounding and is rarely needed after the first tiles.
#include "ops.hpp"

namespace hop {

constexpr int TILE = 128;         // keys of a workgroup's step: 32 a wave
constexpr int DECODE_WGS = 768;   // shares of the line: three workgroups a CU
constexpr float FAR_BELOW = -3.0e38f;
constexpr float LAZY = 8.0f;

struct DecodeArgs {
  herschel_decode_args a;
  herschel_cache c;
  int page_shift;
  int group;     // query heads of a key head
  int rows;      // new tokens * group
  int units;     // key heads * row blocks
  int row_blocks;
  float* part;   // [2 * DECODE_WGS][RB * 16][head_dim + 2]: sums, reference, sum of exponentials
};

// The first tile of a sequence that the window reaches, and its tiles.
__device__ __forceinline__ int first_tile(const DecodeArgs& p, int len) {
  const int lo = p.a.window > 0 ? len - p.a.new_tokens - p.a.window + 1 : 0;
  return lo > 0 ? lo / TILE : 0;
}
__device__ __forceinline__ int seq_len(const DecodeArgs& p, int b, bool report) {
  const int len = p.a.seq_lens[b];
  const int64_t room = p.a.table_stride << p.page_shift;
  const int ok = len < 0 ? 0 : len > room ? (int)room : len;
  if (report && ok != len) flag(p.a.status, HERSCHEL_OP_BAD_LENGTH);
  return ok;
}
// An empty sequence keeps one tile, in which nothing is seen: its rows are written too.
__device__ __forceinline__ int seq_tiles(const DecodeArgs& p, int len) {
  return len > 0 ? (len + TILE - 1) / TILE - first_tile(p, len) : 1;
}

// s_pre[b] = tiles of sequences before b, for all b <= n_seqs; 256 threads.
__device__ __forceinline__ void scan_line(const DecodeArgs& p, int* s_pre, int* s_wave, bool report) {
  const int lane = threadIdx.x % WAVE, wave = threadIdx.x / WAVE;
  int carry = 0;
  for (int b0 = 0; b0 < p.a.n_seqs; b0 += 256) {
    const int b = b0 + threadIdx.x;
    int x = b < p.a.n_seqs ? seq_tiles(p, seq_len(p, b, report)) : 0;
#pragma unroll
    for (int o = 1; o < WAVE; o *= 2) {
      const int y = __shfl_up(x, o);
      if (lane >= o) x += y;
    }
    if (lane == WAVE - 1) s_wave[wave] = x;
    __syncthreads();
    for (int w = 0; w < wave; ++w) x += s_wave[w];
    if (b < p.a.n_seqs) s_pre[b + 1] = carry + x;
    carry += s_wave[0] + s_wave[1] + s_wave[2] + s_wave[3];
    __syncthreads();
  }
  if (threadIdx.x == 0) s_pre[0] = 0;
  __syncthreads();
}

// Share w of a line of U tiles in G shares: [w U / G, (w + 1) U / G).
__device__ __forceinline__ int64_t share_start(int64_t w, int64_t U, int64_t G) { return w * U / G; }
// The share that holds tile x (G <= U, so no share is empty).
__device__ __forceinline__ int64_t share_of(int64_t x, int64_t U, int64_t G) { return ((x + 1) * G - 1) / U; }

template <int TYPE, int KIND, int D, int RB>
__global__ __launch_bounds__(256) void k_decode(DecodeArgs p) {
  // With codes the second product runs in bf16, whose range holds exponential
  // times scale for any scale; for half inputs it runs twice, on the rounded
  // value and on what the rounding left, so that the result keeps half's precision.
  constexpr int PV = quantised(KIND) ? HERSCHEL_BF16 : TYPE;
  constexpr bool SPLIT = quantised(KIND) && TYPE == HERSCHEL_F16;
  constexpr int NS = D / 32;       // steps of the first product
  constexpr int ND = D / 16;       // blocks of dimensions of the second; dimensions of a lane's chunk
  constexpr int CB = code_bytes(KIND);
  extern __shared__ char smem[];
  int* s_pre = (int*)smem;
  float* s_o = (float*)(smem + ((p.a.n_seqs + 1 + 3) & ~3) * 4);  // [4][16][D + 2]
  __shared__ int s_wave[4];

  const int tid = threadIdx.x, lane = tid % WAVE, wave = tid / WAVE, m = lane % 16, g = lane / 16;
  scan_line(p, s_pre, s_wave, blockIdx.x == 0);
  const int64_t U = (int64_t)s_pre[p.a.n_seqs] * p.units, G = U < gridDim.x ? U : gridDim.x;
  if (blockIdx.x >= G) return;
  const int64_t begin = share_start(blockIdx.x, U, G), end = share_start(blockIdx.x + 1, U, G);
  const float to_log2 = p.a.scale * 1.44269504088896340736f;

  for (int64_t pos = begin; pos < end;) {
    // the sequence, unit and tile at this place of the line
    int b = 0;
    for (int n = p.a.n_seqs; n > 1;) {
      const int half = n / 2;
      if ((int64_t)s_pre[b + half] * p.units <= pos) {
        b += half;
        n -= half;
      } else {
        n = half;
      }
    }
    const int len = seq_len(p, b, false), tiles = s_pre[b + 1] - s_pre[b];
    const int64_t rem = pos - (int64_t)s_pre[b] * p.units;
    const int unit = (int)(rem / tiles), tile = (int)(rem % tiles);
    const int n_tiles = (int)min((int64_t)(tiles - tile), end - pos);
    const int head = unit / p.row_blocks, row0 = unit % p.row_blocks * (RB * 16);
    const int32_t* table = p.a.block_table + b * p.a.table_stride;

    // Q: lane (r, g) of block rb holds row r, elements in the order of the keys' chunks;
    // lanes beyond the last row repeat the first one, unused
    u32x4 q[RB][NS];
    int seen_to[RB], seen_from[RB];
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
      const int r = row0 + rb * 16 + m;
      const int tok = r < p.rows ? r / p.group : 0, qh = head * p.group + (r < p.rows ? r % p.group : 0);
      seen_to[rb] = len - p.a.new_tokens + tok + 1;  // keys before this
      seen_from[rb] = p.a.window > 0 ? seen_to[rb] - p.a.window : 0;
      const uint16_t* src = (const uint16_t*)p.a.q + b * p.a.q_seq_stride + tok * p.a.q_strides.row + qh * p.a.q_strides.head;
#pragma unroll
      for (int s = 0; s < NS; ++s) {
        const int d = CB == 2 ? 32 * s + 8 * g : 64 * (s / 2) + 16 * g + 8 * (s & 1);
        q[rb][s] = ((uintptr_t)src & 15) == 0 ? *(const u32x4*)(src + d) : load_elements(src + d);
      }
    }
    f32x4 o[RB][ND];
    float ref[RB], sum[RB];
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
      ref[rb] = FAR_BELOW;
      sum[rb] = 0;
#pragma unroll
      for (int n = 0; n < ND; ++n) o[rb][n] = f32x4{0, 0, 0, 0};
    }
    const int key_begin = (first_tile(p, len) + tile) * TILE, key_end = min(len, key_begin + n_tiles * TILE);
    // keys that every row sees need no mask
    const int all_to = len - p.a.new_tokens + 1, all_from = p.a.window > 0 ? len - p.a.window : 0;

    for (int k0 = key_begin + wave * 32; k0 < key_end; k0 += TILE) {
      // two runs of 16 keys, each within a page; a run past the end reads page 0 unseen
      int64_t run[2];
      bool live[2];
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const int k = k0 + 16 * t;
        int page = k < len ? table[k >> p.page_shift] : 0;
        live[t] = k < len && page >= 0 && page < p.c.n_pages;
        if (k < len && !live[t] && lane == 0) flag(p.a.status, HERSCHEL_OP_BAD_PAGE);
        if (!live[t]) page = 0;
        run[t] = (((int64_t)page * p.c.n_heads + head) << p.page_shift) + (live[t] ? k & (p.c.page_size - 1) : 0);
      }
      // loads: keys, then values, then scales
      u32x4 kf[2][CB == 2 ? NS : NS / 2];
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const char* kp = (const char*)p.c.k + (run[t] + m) * (D * CB) + 16 * g;
#pragma unroll
        for (int s = 0; s < (CB == 2 ? NS : NS / 2); ++s) kf[t][s] = *(const u32x4*)(kp + 64 * s);
      }
      uint32_t vf[8][ND / 2 * CB / 2];  // eight keys, ND dimensions each
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const char* vp = (const char*)p.c.v + (run[j / 4] + 4 * g + j % 4) * (D * CB) + m * (ND * CB);
        constexpr int W = ND / 2 * CB / 2;
        if constexpr (W == 4) {
          const u32x4 x = *(const u32x4*)vp;
          vf[j][0] = x[0], vf[j][1] = x[1], vf[j][2] = x[2], vf[j][3] = x[3];
        } else if constexpr (W == 2) {
          const u32x2 x = *(const u32x2*)vp;
          vf[j][0] = x[0], vf[j][1] = x[1];
        } else {
          vf[j][0] = *(const uint32_t*)vp;
        }
      }
      f32x4 ks[2], vs[2];
      if constexpr (quantised(KIND)) {
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          ks[t] = *(const f32x4*)(p.c.k_scale + run[t] + 4 * g);
          vs[t] = *(const f32x4*)(p.c.v_scale + run[t] + 4 * g);
        }
      }

      // S^T = K Q^T
      f32x4 sc[RB][2];
#pragma unroll
      for (int rb = 0; rb < RB; ++rb)
#pragma unroll
        for (int t = 0; t < 2; ++t) sc[rb][t] = f32x4{0, 0, 0, 0};
#pragma unroll
      for (int t = 0; t < 2; ++t) {
#pragma unroll
        for (int s = 0; s < NS; ++s) {
          u32x4 ka;
          if constexpr (!quantised(KIND)) {
            ka = kf[t][s];
          } else {
            const uint32_t w0 = kf[t][s / 2][2 * (s & 1)], w1 = kf[t][s / 2][2 * (s & 1) + 1];
            ka = u32x4{decode2<KIND, TYPE, false>(w0), decode2<KIND, TYPE, true>(w0), decode2<KIND, TYPE, false>(w1),
                       decode2<KIND, TYPE, true>(w1)};
          }
#pragma unroll
          for (int rb = 0; rb < RB; ++rb) sc[rb][t] = mfma16<TYPE>(ka, q[rb][s], sc[rb][t]);
        }
      }
      // V^T: pairs of keys of one dimension
      u32x4 vt[ND];
#pragma unroll
      for (int j = 0; j < 4; ++j) {  // keys 2 j, 2 j + 1
#pragma unroll
        for (int d = 0; d < ND / 2; ++d) {
          uint32_t x, y;
          if constexpr (!quantised(KIND)) {
            x = vf[2 * j][d];
            y = vf[2 * j + 1][d];
          } else if (d & 1) {
            x = decode2<KIND, PV, true>(vf[2 * j][d / 2]);
            y = decode2<KIND, PV, true>(vf[2 * j + 1][d / 2]);
          } else {
            x = decode2<KIND, PV, false>(vf[2 * j][d / 2]);
            y = decode2<KIND, PV, false>(vf[2 * j + 1][d / 2]);
          }
          vt[2 * d][j] = __builtin_amdgcn_perm(y, x, 0x05040100);
          vt[2 * d + 1][j] = __builtin_amdgcn_perm(y, x, 0x07060302);
        }
      }
      const bool edge = k0 + 32 > all_to || k0 < all_from || !live[0] || !live[1];
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) {
        float x[8];
        uint32_t seen = 0xff;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          float f = sc[rb][i / 4][i % 4] * to_log2;
          if constexpr (quantised(KIND)) f *= ks[i / 4][i % 4];
          x[i] = f;
        }
        if (edge) {
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const int key = k0 + 16 * (i / 4) + 4 * g + i % 4;
            if (!(live[i / 4] && key < seen_to[rb] && key >= seen_from[rb])) {
              x[i] = -INFINITY;
              seen &= ~(1u << i);
            }
          }
        }
        float top = fmaxf(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])), fmaxf(fmaxf(x[4], x[5]), fmaxf(x[6], x[7])));
        if (__ballot(top > ref[rb] + LAZY)) {
          top = fmaxf(top, __shfl_xor(top, 16));
          top = fmaxf(top, __shfl_xor(top, 32));
          const float to = fmaxf(ref[rb], top), by = __builtin_amdgcn_exp2f(ref[rb] - to);
          ref[rb] = to;
          sum[rb] *= by;
#pragma unroll
          for (int n = 0; n < ND; ++n) o[rb][n] *= by;
        }
        float e[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          e[i] = __builtin_amdgcn_exp2f(x[i] - ref[rb]);
          sum[rb] += e[i];
          if constexpr (quantised(KIND)) e[i] = (seen >> i) & 1 ? e[i] * vs[i / 4][i % 4] : 0.0f;
        }
        u32x4 pb, pl;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          pb[i] = pack2<PV>(e[2 * i], e[2 * i + 1]);
          if constexpr (SPLIT) {
            float r0, r1;
            unpack2<PV>(pb[i], r0, r1);
            pl[i] = pack2<PV>(e[2 * i] - r0, e[2 * i + 1] - r1);
          }
        }
        if (!edge) {
#pragma unroll
          for (int n = 0; n < ND; ++n) {
            o[rb][n] = mfma16<PV>(vt[n], pb, o[rb][n]);
            if constexpr (SPLIT) o[rb][n] = mfma16<PV>(vt[n], pl, o[rb][n]);
          }
        } else {
          // a value that is not finite must reach the rows that see its key and
          // no other: it is taken out of the product, and added where seen
          constexpr uint32_t ONE = PV == HERSCHEL_BF16 ? 0x3f80u : 0x3c00u;
          constexpr uint32_t INF = PV == HERSCHEL_BF16 ? 0x7f80u : 0x7c00u;
          u32x4 sees;
#pragma unroll
          for (int i = 0; i < 4; ++i)
            sees[i] = ((seen >> (2 * i)) & 1 ? ONE : 0u) | ((seen >> (2 * i + 1)) & 1 ? ONE << 16 : 0u);
#pragma unroll
          for (int n = 0; n < ND; ++n) {
            u32x4 bad, va;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              bad[i] = not_finite2<PV>(vt[n][i]);
              va[i] = vt[n][i] & ~bad[i];
            }
            o[rb][n] = mfma16<PV>(va, pb, o[rb][n]);
            if constexpr (SPLIT) o[rb][n] = mfma16<PV>(va, pl, o[rb][n]);
            if (__ballot((bad[0] | bad[1] | bad[2] | bad[3]) != 0)) {
              u32x4 up, down;  // +infinity or NaN, -infinity or NaN
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                const uint32_t w = vt[n][i];
                uint32_t u = 0, d = 0;
#pragma unroll
                for (int h = 0; h < 32; h += 16) {
                  const uint32_t z = (w >> h) & 0xffffu;
                  if ((bad[i] >> h) & 1) {
                    if (z != (INF | 0x8000u)) u |= ONE << h;
                    if (z != INF) d |= ONE << h;
                  }
                }
                up[i] = u;
                down[i] = d;
              }
              const f32x4 nu = mfma16<PV>(up, sees, f32x4{0, 0, 0, 0}), nd = mfma16<PV>(down, sees, f32x4{0, 0, 0, 0});
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                if (nu[i] > 0) o[rb][n][i] += INFINITY;
                if (nd[i] > 0) o[rb][n][i] -= INFINITY;
              }
            }
          }
        }
      }
    }

    // The four waves' parts of these rows, joined through LDS block by block.
    const bool whole = tile == 0 && n_tiles == tiles;
    const int64_t slot = 2 * (int64_t)blockIdx.x + (pos == begin ? 0 : 1);
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
      float s = sum[rb];
      s += __shfl_xor(s, 16);
      s += __shfl_xor(s, 32);
      __syncthreads();
      float* mine = s_o + wave * 16 * (D + 2) + m * (D + 2);
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int n = 0; n < ND; ++n) mine[ND * (4 * g + i) + n] = o[rb][n][i];  // dimension ND (4 g + i) + n
      if (g == 0) {
        mine[D] = ref[rb];
        mine[D + 1] = s;
      }
      __syncthreads();
      // 16 rows by 16 lanes, ND dimensions each
      const int r = row0 + rb * 16 + tid / 16, d0 = tid % 16 * ND;
      if (r < p.rows) {
        const float* all = s_o + tid / 16 * (D + 2);
        constexpr int WS = 16 * (D + 2);
        const float top = fmaxf(fmaxf(all[D], all[WS + D]), fmaxf(all[2 * WS + D], all[3 * WS + D]));
        float acc[ND], den = 0;
#pragma unroll
        for (int n = 0; n < ND; ++n) acc[n] = 0;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          const float by = __builtin_amdgcn_exp2f(all[w * WS + D] - top);
          den += all[w * WS + D + 1] * by;
#pragma unroll
          for (int n = 0; n < ND; ++n) acc[n] += all[w * WS + d0 + n] * by;
        }
        if (whole) {
          const float inv = den > 0 ? 1.0f / den : den == 0 ? 0.0f : den;  // no key seen: 0; NaN stays
          const int64_t at = ((int64_t)b * p.a.new_tokens + r / p.group) * p.a.q_heads + head * p.group + r % p.group;
          uint32_t* out = (uint32_t*)((uint16_t*)p.a.out + at * D + d0);
#pragma unroll
          for (int n = 0; n < ND; n += 2) out[n / 2] = pack2<TYPE>(acc[n] * inv, acc[n + 1] * inv);
          if (p.a.lse && tid % 16 == 0)
            p.a.lse[at] = den == 0 ? -INFINITY : (top + __builtin_amdgcn_logf(den)) * 0.69314718055994530942f;
        } else {
          float* to = p.part + (slot * (RB * 16) + rb * 16 + tid / 16) * (D + 2);
#pragma unroll
          for (int n = 0; n < ND; ++n) to[d0 + n] = acc[n];
          if (tid % 16 == 0) {
            to[D] = top;
            to[D + 1] = den;
          }
        }
      }
    }
    pos += n_tiles;
  }
}

// Joins the parts of each sequence's head that more than one share holds: a
// workgroup per (sequence, unit), 16 lanes a row.
template <int TYPE, int D, int RB>
__global__ __launch_bounds__(256) void k_decode_join(DecodeArgs p) {
  extern __shared__ char smem[];
  int* s_pre = (int*)smem;
  __shared__ int s_wave[4];
  constexpr int ND = D / 16;
  scan_line(p, s_pre, s_wave, false);
  const int b = blockIdx.x / p.units, unit = blockIdx.x % p.units, tiles = s_pre[b + 1] - s_pre[b];
  const int64_t U = (int64_t)s_pre[p.a.n_seqs] * p.units, G = U < DECODE_WGS ? U : DECODE_WGS;
  const int64_t at0 = (int64_t)s_pre[b] * p.units + (int64_t)unit * tiles;
  const int64_t first = share_of(at0, U, G), last = share_of(at0 + tiles - 1, U, G);
  if (first == last) return;
  const int head = unit / p.row_blocks, row0 = unit % p.row_blocks * (RB * 16);
  const int d0 = threadIdx.x % 16 * ND;
  for (int rr = threadIdx.x / 16; rr < RB * 16; rr += 16) {
    const int r = row0 + rr;
    if (r >= p.rows) continue;
    float top = FAR_BELOW, den = 0, acc[ND];
#pragma unroll
    for (int n = 0; n < ND; ++n) acc[n] = 0;
    for (int64_t w = first; w <= last; ++w) {
      const int64_t slot = 2 * w + (w == first && share_start(w, U, G) != at0 ? 1 : 0);
      const float* from = p.part + (slot * (RB * 16) + rr) * (D + 2);
      const float t = from[D], to = fmaxf(top, t);
      const float old = __builtin_amdgcn_exp2f(top - to), by = __builtin_amdgcn_exp2f(t - to);
      den = den * old + from[D + 1] * by;
#pragma unroll
      for (int n = 0; n < ND; ++n) acc[n] = acc[n] * old + from[d0 + n] * by;
      top = to;
    }
    const float inv = den > 0 ? 1.0f / den : den == 0 ? 0.0f : den;
    const int64_t at = ((int64_t)b * p.a.new_tokens + r / p.group) * p.a.q_heads + head * p.group + r % p.group;
    uint32_t* out = (uint32_t*)((uint16_t*)p.a.out + at * D + d0);
#pragma unroll
    for (int n = 0; n < ND; n += 2) out[n / 2] = pack2<TYPE>(acc[n] * inv, acc[n + 1] * inv);
    if (p.a.lse && threadIdx.x % 16 == 0)
      p.a.lse[at] = den == 0 ? -INFINITY : (top + __builtin_amdgcn_logf(den)) * 0.69314718055994530942f;
  }
}

template <int TYPE, int KIND, int D, int RB>
static int decode_launch(DecodeArgs& p) {
  const size_t pre = ((p.a.n_seqs + 1 + 3) & ~3) * 4;
  const int rc = launch(k_decode<TYPE, KIND, D, RB>, dim3(DECODE_WGS), dim3(256), pre + 4 * 16 * (D + 2) * 4,
                        p.a.hip_stream, p);
  if (rc != HERSCHEL_OK) return rc;
  return launch(k_decode_join<TYPE, D, RB>, dim3((unsigned)(p.a.n_seqs * p.units)), dim3(256), pre, p.a.hip_stream, p);
}

template <int TYPE, int KIND>
static int decode_size(DecodeArgs& p) {
  if (p.c.head_dim == 64) return p.rows <= 16 ? decode_launch<TYPE, KIND, 64, 1>(p) : decode_launch<TYPE, KIND, 64, 2>(p);
  return p.rows <= 16 ? decode_launch<TYPE, KIND, 128, 1>(p) : decode_launch<TYPE, KIND, 128, 2>(p);
}

// Rows of a workgroup: one block of 16 columns of the matrix products, or two.
static int decode_rows(int rows) { return rows <= 16 ? 16 : 32; }

static bool decode_sizes_ok(int32_t n_seqs, int32_t new_tokens, int32_t q_heads, const herschel_cache* c) {
  return cache_ok(c) && (c->head_dim == 64 || c->head_dim == 128) && n_seqs >= 1 &&
         n_seqs <= HERSCHEL_MAX_DECODE_SEQS && new_tokens >= 1 && new_tokens <= 1024 && q_heads >= 1 &&
         q_heads <= (1 << 14) && q_heads % c->n_heads == 0;
}

}  // namespace hop

extern "C" int herschel_attn_decode_workspace(int32_t n_seqs, int32_t new_tokens, int32_t q_heads,
                                              const herschel_cache* cache, size_t* bytes) {
  using namespace hop;
  if (!bytes || !decode_sizes_ok(n_seqs, new_tokens, q_heads, cache)) return HERSCHEL_EINVAL;
  *bytes = (size_t)2 * DECODE_WGS * decode_rows(new_tokens * (q_heads / cache->n_heads)) * (cache->head_dim + 2) * 4;
  return HERSCHEL_OK;
}

extern "C" int herschel_attn_decode(const herschel_decode_args* args, const herschel_cache* cache) {
  using namespace hop;
  if (!args) return HERSCHEL_EINVAL;
  const herschel_decode_args& a = *args;
  size_t need = 0;
  if (herschel_attn_decode_workspace(a.n_seqs, a.new_tokens, a.q_heads, cache, &need) != HERSCHEL_OK) return HERSCHEL_EINVAL;
  if (!a.q || !a.out || !aligned(a.q, 2) || !aligned(a.out, 16) || !a.seq_lens || a.table_stride < 0) return HERSCHEL_EINVAL;
  if (!a.block_table && a.table_stride) return HERSCHEL_EINVAL;
  if (!type_ok(a.type) || !strides_ok(a.q_strides) || a.q_seq_stride < 0 || a.window < 0 || !isfinite(a.scale))
    return HERSCHEL_EINVAL;
  if (!quantised(cache->kind) && cache->kind != a.type) return HERSCHEL_EINVAL;
  if (!a.workspace || !aligned(a.workspace, 256) || a.workspace_bytes < need) return HERSCHEL_EWORKSPACE;
  DecodeArgs p{};
  p.a = a;
  p.c = *cache;
  p.page_shift = log2i(cache->page_size);
  p.group = a.q_heads / cache->n_heads;
  p.rows = a.new_tokens * p.group;
  const int block = decode_rows(p.rows);
  p.row_blocks = (p.rows + block - 1) / block;
  p.units = cache->n_heads * p.row_blocks;
  p.part = (float*)a.workspace;
  const bool bf = a.type == HERSCHEL_BF16;
  switch (cache->kind) {
    case HERSCHEL_FP8:
      return bf ? decode_size<HERSCHEL_BF16, HERSCHEL_FP8>(p) : decode_size<HERSCHEL_F16, HERSCHEL_FP8>(p);
    case HERSCHEL_INT8:
      return bf ? decode_size<HERSCHEL_BF16, HERSCHEL_INT8>(p) : decode_size<HERSCHEL_F16, HERSCHEL_INT8>(p);
    default:
      return bf ? decode_size<HERSCHEL_BF16, HERSCHEL_BF16>(p) : decode_size<HERSCHEL_F16, HERSCHEL_F16>(p);
  }
}
