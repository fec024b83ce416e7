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
//  - A step's 16 KB (8 with codes) a wave are asked for at once; the waits are
//    filled by the other waves of the SIMD.  (When tried, loading the next step's
//    rows before this one was worked on cost registers, and with them waves: 105 us
//    became 110 for 32 requests of 4096 tokens in bf16, 92 became 102 for 64 in fp8.
//    Its keys once the scores are there and its values after the second product spilled
//    with fp8, 79 became 136 us, and gained nothing with int8, 52 became 54.)
//  - The second kernel costs 4 to 7 us.  Joining in the first, by the workgroup
//    whose part is the last one there, cost more when tried: parts written through the
//    caches to where all XCDs see them 14.0 us against 12.9 for one request of 4000
//    tokens, 140 against 121 for three long contexts.
//
// 64 requests of 512 to 8704 tokens in fp8, 396 MB: 79 us, 5.0 TB/s, a copy's rate.
// One of 4000 tokens in bf16, 16 MB: 13.0 us, two kernels' latency.  Four drafted
// tokens of three long contexts in int8, 473 MB: 107 to 110 us, 4.4 TB/s; with 20 rows of
// 32 in use, codes that become halves and every product of the second kind done
// twice, vector instructions take half of that.
//
// The reference of a row's exponentials moves only when a step's sum shows that
// it does not fit (ops.hpp); no maximum is computed otherwise.  Rows of keys beyond
// the sequence's end, or before all windows, are never read: a hidden key of a
// step stands at a seen one's row, with the exponential 0.  An infinity or a NaN
// times that 0 is a NaN, and so is an infinity whose weight is too small for 32
// bits: a wave whose sums are not finite goes over its keys once more, with such
// values taken out of the products and added to the rows that see them.
#include <type_traits>

#include "ops.hpp"

namespace hop {

#define INLINE __attribute__((always_inline))

constexpr int TILE = 128;         // keys of a workgroup's step: 32 a wave
// Shares of the line: as many workgroups as the CUs hold, by registers.  Of heads
// of 128 three a CU with codes and one row block (64 requests in fp8 80 us against
// 83 with two), else two (bf16 73 and 73 us; more with two blocks spill: 120 us
// become 257).  A step of heads of 64 has half the bytes to wait for and fewer
// registers: four (64 requests in int8 52 us against 54 with three, in fp8 53
// against 52), with two row blocks of codes three (three long contexts 72 against
// 79 with two and 109 with four).
constexpr int MAX_SHARES = 1024;
constexpr int shares_of_cu(int kind, int row_blocks, int dim) {
  return dim == 64 ? (row_blocks == 1 ? 4 : quantised(kind) ? 3 : 2) : quantised(kind) && row_blocks == 1 ? 3 : 2;
}
constexpr float FAR_BELOW = -3.0e38f;

struct DecodeArgs {
  herschel_decode_args a;
  herschel_cache c;
  int page_shift;
  int group;     // query heads of a key head
  int rows;      // new tokens * group
  int units;     // key heads * row blocks
  int row_blocks;
  bool q_vec;    // Q's chunks of 16 bytes are aligned
  int2* span;    // [n_seqs * units] first part and last share of a row block; first part -1: nothing to join
  float* part;   // [2 * MAX_SHARES][RB * 16][head_dim + 2]: sums, reference, sum of exponentials
};

// The first tile of a sequence that the window reaches, and its tiles.
__device__ __forceinline__ int first_tile(const DecodeArgs& p, int len) {
  return window_from(len - p.a.new_tokens, p.a.window) / TILE;
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
  if (p.a.n_seqs <= WAVE) {
    if (wave == 0) {
      int x = lane < p.a.n_seqs ? seq_tiles(p, seq_len(p, lane, report)) : 0;
#pragma unroll
      for (int o = 1; o < WAVE; o *= 2) {
        const int y = __shfl_up(x, o);
        if (lane >= o) x += y;
      }
      if (lane < p.a.n_seqs) s_pre[lane + 1] = x;
      if (lane == 0) s_pre[0] = 0;
    }
    __syncthreads();
    return;
  }
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

// Factor of sums whose reference moves; of none, which are 0, 1.
__device__ __forceinline__ float factor(float from, float to) {
  return from > FAR_BELOW ? __builtin_amdgcn_exp2f(from - to) : 1.0f;
}

// a / b of numbers that are not negative: a 64-bit division takes a microsecond.
__device__ __forceinline__ int64_t divide(int64_t a, int64_t b) {
  return ((uint64_t)(a | b) >> 32) == 0 ? (int64_t)((uint32_t)a / (uint32_t)b) : a / b;
}
// Share w of a line of U tiles in G shares: [w U / G, (w + 1) U / G).
__device__ __forceinline__ int64_t share_start(int64_t w, int64_t U, int64_t G) { return divide(w * U, G); }
// The share that holds tile x (G <= U, so no share is empty).
__device__ __forceinline__ int64_t share_of(int64_t x, int64_t U, int64_t G) { return divide((x + 1) * G - 1, U); }

template <int TYPE, int KIND, int D, int RB>
__global__ __launch_bounds__(256, shares_of_cu(KIND, RB, D)) void k_decode(DecodeArgs p) {
  // With codes the second product runs in bf16, whose range holds exponential
  // times scale for any scale.  It runs twice, on the rounded value and on what the
  // rounding left, so that the result keeps the rows' precision: with one row block
  // that is hidden behind the reads (64 requests of bf16 rows in fp8 80.5 against
  // 81.2 us and 0.0017 from 64 bits instead of 0.0023, 32 in a bf16 cache 72.6
  // against 73.2).  With two it takes 8% (three long contexts in fp8 99 against 107
  // us): there rows of the cache's type and bf16 rows, whose own rounding is as large,
  // take the rounded value alone; half rows over codes, whose rounding is finer than
  // bf16's, do not.
  constexpr int PV = quantised(KIND) ? HERSCHEL_BF16 : TYPE;
  constexpr bool SPLIT = RB == 1 || (quantised(KIND) && TYPE == HERSCHEL_F16);
  constexpr int NS = D / 32;       // steps of the first product
  constexpr int ND = D / 16;       // blocks of dimensions of the second; dimensions of a lane's chunk
  constexpr int CB = code_bytes(KIND);
  constexpr int VW = ND / 2 * CB / 2;  // words of a lane's chunk of V
  extern __shared__ char smem[];
  int* s_pre = (int*)smem;
  float* s_o = (float*)(smem + ((p.a.n_seqs + 1 + 3) & ~3) * 4);  // [4][16][D + 2]
  __shared__ int s_wave[4];

  const int tid = threadIdx.x, lane = tid % WAVE, wave = __builtin_amdgcn_readfirstlane(tid / WAVE), m = lane % 16, g = lane / 16;
  scan_line(p, s_pre, s_wave, blockIdx.x == 0);
  auto uniform = [](int x) INLINE { return __builtin_amdgcn_readfirstlane(x); };  // what came through LDS
  const int64_t U = (int64_t)uniform(s_pre[p.a.n_seqs]) * p.units, G = U < gridDim.x ? U : gridDim.x;
  if (blockIdx.x >= G) return;
  const int64_t begin = share_start(blockIdx.x, U, G), end = share_start(blockIdx.x + 1, U, G);
  const uint32_t n_pages = (uint32_t)min(p.c.n_pages, (int64_t)INT32_MAX + 1);
  const float to_log2 = p.a.scale * 1.44269504088896340736f;

  for (int64_t pos = begin; pos < end;) {
    // the sequence, unit and tile at this place of the line
    int b = 0;
    for (int n = p.a.n_seqs; n > 1;) {
      const int half = n / 2;
      if ((int64_t)uniform(s_pre[b + half]) * p.units <= pos) {
        b += half;
        n -= half;
      } else {
        n = half;
      }
    }
    const int before = uniform(s_pre[b]), tiles = uniform(s_pre[b + 1]) - before, len = uniform(seq_len(p, b, false));
    const int64_t rem = pos - (int64_t)before * p.units;
    const int unit = (int)divide(rem, tiles), tile = (int)(rem - (int64_t)unit * tiles);
    const int n_tiles = (int)min((int64_t)(tiles - tile), end - pos);
    const int head = unit / p.row_blocks, row0 = unit % p.row_blocks * (RB * 16);
    // through the scalar cache: a page id is the whole wave's
    typedef const __attribute__((address_space(4))) int32_t Table;
    Table* table = (Table*)(uintptr_t)(p.a.block_table + b * p.a.table_stride);

    const int key_begin = (first_tile(p, len) + tile) * TILE, key_end = min(len, key_begin + n_tiles * TILE);
    // keys that every row sees need no mask; those that some row sees are read
    const int all_to = len - p.a.new_tokens + 1, all_from = window_from(len - 1, p.a.window);
    const int any_from = window_from(len - p.a.new_tokens, p.a.window);

    struct Step {
      u32x4 k[2][CB == 2 ? NS : NS / 2];
      uint32_t v[8][VW];  // eight keys, ND dimensions each
      f32x4 ks[2], vs[2];
      bool live[2];
    };
    // page ids of the two runs of 16 keys of a step, each within a page
    auto find = [&](int k0, int (&page)[2]) INLINE {
#pragma unroll
      for (int t = 0; t < 2; ++t) page[t] = table[min(max(k0 + 16 * t, any_from), len - 1) >> p.page_shift];
    };
    // All that the first step waits for is asked for in one go: page ids, Q, rows.
    int k0 = key_begin + wave * 32, page[2] = {0, 0};
    if (k0 < key_end) find(k0, page);
    // Q: lane (r, g) of block rb holds row r, elements in the order of the keys' chunks;
    // lanes beyond the last row repeat the first one, unused
    u32x4 q[RB][NS];
    int seen_to[RB], seen_from[RB];
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
      const int r = row0 + rb * 16 + m;
      const int tok = r < p.rows ? r / p.group : 0, qh = head * p.group + (r < p.rows ? r % p.group : 0);
      seen_to[rb] = len - p.a.new_tokens + tok + 1;  // keys before this
      seen_from[rb] = window_from(seen_to[rb] - 1, p.a.window);
      const uint16_t* src = (const uint16_t*)p.a.q + b * p.a.q_seq_stride + tok * p.a.q_strides.row + qh * p.a.q_strides.head;
#pragma unroll
      for (int s = 0; s < NS; ++s) {
        const int d = CB == 2 ? 32 * s + 8 * g : 64 * (s / 2) + 16 * g + 8 * (s & 1);
        q[rb][s] = p.q_vec ? *(const u32x4*)(src + d) : load_elements(src + d);
      }
    }
    f32x4 o[RB][ND];
    float ref[RB], sum[RB];
    bool apart = false;  // values that are not finite are kept out of the products
    // A lane's places in a run of 16 keys: its key's row, the first of its four values' rows, their scales.
    const uint32_t koff = m * (D * CB) + 16 * g, voff = 4 * g * (D * CB) + m * (ND * CB), soff = 4 * g;
    auto load_v = [&](uint32_t* to, const char* from) INLINE {  // whole rows, read once: past the caches (32 x 4096 in bf16 102 to 93 us)
      if constexpr (VW == 4) {
        const u32x4 x = __builtin_nontemporal_load((const u32x4*)from);
        to[0] = x[0], to[1] = x[1], to[2] = x[2], to[3] = x[3];
      } else if constexpr (VW == 2) {
        const u32x2 x = __builtin_nontemporal_load((const u32x2*)from);
        to[0] = x[0], to[1] = x[1];
      } else {
        to[0] = *(const uint32_t*)from;
      }
    };
    auto load = [&](Step& s, int k0, const int (&page)[2]) INLINE {
      const bool inside = k0 >= any_from && k0 + 32 <= len;
      const int in_page = p.c.page_size - 1;
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        s.live[t] = (uint32_t)page[t] < n_pages;
        const int id = uniform(s.live[t] ? page[t] : 0);  // the wave's, also where one lane reports
        if (!s.live[t] && lane == 0) flag(p.a.status, HERSCHEL_OP_BAD_PAGE);
        const int64_t base = ((int64_t)id * p.c.n_heads + head) << p.page_shift;
        const int k = k0 + 16 * t;
        if (inside) {  // addresses of the wave, offsets of the lane: nothing to compute
          const int64_t at = base + (k & in_page);
          const char *kp = (const char*)p.c.k + at * (D * CB), *vp = (const char*)p.c.v + at * (D * CB);
#pragma unroll
          for (int i = 0; i < (CB == 2 ? NS : NS / 2); ++i) s.k[t][i] = *(const u32x4*)(kp + koff + 64 * i);
#pragma unroll
          for (int j = 0; j < 4; ++j) load_v(s.v[4 * t + j], vp + voff + j * (D * CB));
          if constexpr (quantised(KIND)) {
            s.ks[t] = *(const f32x4*)(p.c.k_scale + at + soff);
            s.vs[t] = *(const f32x4*)(p.c.v_scale + at + soff);
          }
        } else {
          auto row = [&](int key) INLINE { return base + (min(max(key, any_from), len - 1) & in_page); };
          const char* kp = (const char*)p.c.k + row(k + m) * (D * CB) + 16 * g;
#pragma unroll
          for (int i = 0; i < (CB == 2 ? NS : NS / 2); ++i) s.k[t][i] = *(const u32x4*)(kp + 64 * i);
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const int64_t at = row(k + 4 * g + j);
            load_v(s.v[4 * t + j], (const char*)p.c.v + at * (D * CB) + m * (ND * CB));
            if constexpr (quantised(KIND)) {
              s.ks[t][j] = p.c.k_scale[at];
              s.vs[t][j] = p.c.v_scale[at];
            }
          }
        }
      }
    };
    // Factor of sums whose reference moves.  0 times an infinity would be a NaN: the second pass starts from the first's
    // last reference, from which bf16's goes up by a few powers of two at most, and a half times 2^-126 is nothing.
    auto moved_by = [](float from, float to) INLINE {
      const float by = __builtin_amdgcn_exp2f(from - to);
      return PV == HERSCHEL_F16 ? fmaxf(by, 0x1p-126f) : by;
    };
    auto work = [&](Step& s, int k0) INLINE {
      // S^T = K Q^T
      f32x4 sc[RB][2];
#pragma unroll
      for (int rb = 0; rb < RB; ++rb)
#pragma unroll
        for (int t = 0; t < 2; ++t) sc[rb][t] = f32x4{0, 0, 0, 0};
#pragma unroll
      for (int t = 0; t < 2; ++t) {
#pragma unroll
        for (int i = 0; i < NS; ++i) {
          u32x4 ka;
          if constexpr (!quantised(KIND)) {
            ka = s.k[t][i];
          } else {
            const uint32_t w0 = s.k[t][i / 2][2 * (i & 1)], w1 = s.k[t][i / 2][2 * (i & 1) + 1];
            ka = u32x4{decode2<KIND, TYPE, false>(w0), decode2<KIND, TYPE, true>(w0), decode2<KIND, TYPE, false>(w1),
                       decode2<KIND, TYPE, true>(w1)};
          }
#pragma unroll
          for (int rb = 0; rb < RB; ++rb) sc[rb][t] = mfma16<TYPE>(ka, q[rb][i], sc[rb][t]);
        }
      }
      const bool edge = k0 + 32 > all_to || k0 < all_from || !s.live[0] || !s.live[1];
      float f[8];  // of the scores: to powers of two, times the key's scale
#pragma unroll
      for (int i = 0; i < 8; ++i) f[i] = quantised(KIND) ? to_log2 * s.ks[i / 4][i % 4] : to_log2;
      u32x4 pb[RB], pl[RB];
      uint32_t seen[RB];
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) {
        seen[rb] = 0xff;
        if (edge) {
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const int key = k0 + 16 * (i / 4) + 4 * g + i % 4;
            if (!(s.live[i / 4] && key < seen_to[rb] && key >= seen_from[rb])) seen[rb] &= ~(1u << i);
          }
        }
        float e[8];
        auto exponentials = [&]() INLINE {
          float t = 0;
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            e[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[rb][i / 4][i % 4], f[i], -ref[rb]));
            if (edge) e[i] = (seen[rb] >> i) & 1 ? e[i] : 0.0f;
            t += e[i];
          }
          return t;
        };
        float t = exponentials();
        if (Reference<PV>::template off<4>(t)) {
          float top = FAR_BELOW;
#pragma unroll
          for (int i = 0; i < 8; ++i) top = fmaxf(top, (seen[rb] >> i) & 1 ? sc[rb][i / 4][i % 4] * f[i] : FAR_BELOW);
          top = fmaxf(top, __shfl_xor(top, 16));
          top = fmaxf(top, __shfl_xor(top, 32));
          float total = sum[rb] + __shfl_xor(sum[rb], 16);
          total += __shfl_xor(total, 32);
          const float to = Reference<PV>::moved(ref[rb], top, total), by = moved_by(ref[rb], to);
          ref[rb] = to;
          sum[rb] *= by;
#pragma unroll
          for (int n = 0; n < ND; ++n) o[rb][n] *= by;
          t = exponentials();
        }
        sum[rb] += t;
        if constexpr (quantised(KIND)) {
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            e[i] *= s.vs[i / 4][i % 4];
            if (edge) e[i] = (seen[rb] >> i) & 1 ? e[i] : 0.0f;
          }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          pb[rb][i] = pack2<PV>(e[2 * i], e[2 * i + 1]);
          if constexpr (SPLIT) {
            float r0, r1;
            unpack2<PV>(pb[rb][i], r0, r1);
            pl[rb][i] = pack2<PV>(e[2 * i] - r0, e[2 * i + 1] - r1);
          }
        }
      }
      // O^T += V^T P^T, two dimensions of a lane's chunk at a time: V^T has pairs of keys of one dimension
#pragma unroll
      for (int d = 0; d < ND / 2; ++d) {
        u32x4 vt[2];
#pragma unroll
        for (int j = 0; j < 4; ++j) {  // keys 2 j, 2 j + 1
          uint32_t x, y;
          if constexpr (!quantised(KIND)) {
            x = s.v[2 * j][d];
            y = s.v[2 * j + 1][d];
          } else if (d & 1) {
            x = decode2<KIND, PV, true>(s.v[2 * j][d / 2]);
            y = decode2<KIND, PV, true>(s.v[2 * j + 1][d / 2]);
          } else {
            x = decode2<KIND, PV, false>(s.v[2 * j][d / 2]);
            y = decode2<KIND, PV, false>(s.v[2 * j + 1][d / 2]);
          }
          vt[0][j] = __builtin_amdgcn_perm(y, x, 0x05040100);
          vt[1][j] = __builtin_amdgcn_perm(y, x, 0x07060302);
        }
        // A value that is not finite must reach the rows that see its key, and no other.
        if (KIND != HERSCHEL_INT8 && apart) {
          constexpr uint32_t ONE = PV == HERSCHEL_BF16 ? 0x3f80u : 0x3c00u;
          constexpr uint32_t INF = PV == HERSCHEL_BF16 ? 0x7f80u : 0x7c00u;
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            u32x4 up, down, rest;  // +infinity or NaN, -infinity or NaN, finite
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const uint32_t w = vt[h][i], bad = not_finite2<PV>(w);
              up[i] = down[i] = 0;
#pragma unroll
              for (int z = 0; z < 32; z += 16) {
                const uint32_t x = (w >> z) & 0xffffu;
                if ((bad >> z) & 1) {
                  if (x != (INF | 0x8000u)) up[i] |= ONE << z;
                  if (x != INF) down[i] |= ONE << z;
                }
              }
              rest[i] = w & ~bad;
            }
            vt[h] = rest;
            if (__ballot((up[0] | up[1] | up[2] | up[3] | down[0] | down[1] | down[2] | down[3]) != 0)) {
#pragma unroll
              for (int rb = 0; rb < RB; ++rb) {
                u32x4 sees;
#pragma unroll
                for (int i = 0; i < 4; ++i)
                  sees[i] = ((seen[rb] >> (2 * i)) & 1 ? ONE : 0u) | ((seen[rb] >> (2 * i + 1)) & 1 ? ONE << 16 : 0u);
                const f32x4 zero = {0, 0, 0, 0}, nu = mfma16<PV>(up, sees, zero), nd = mfma16<PV>(down, sees, zero);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                  if (nu[i] > 0) o[rb][2 * d + h][i] += INFINITY;
                  if (nd[i] > 0) o[rb][2 * d + h][i] -= INFINITY;
                }
              }
            }
          }
        }
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int rb = 0; rb < RB; ++rb) {
            o[rb][2 * d + h] = mfma16<PV>(vt[h], pb[rb], o[rb][2 * d + h]);
            if constexpr (SPLIT) o[rb][2 * d + h] = mfma16<PV>(vt[h], pl[rb], o[rb][2 * d + h]);
          }
      }
    };
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) ref[rb] = FAR_BELOW;
    Step s;
    for (;;) {
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) {
        sum[rb] = 0;
#pragma unroll
        for (int n = 0; n < ND; ++n) o[rb][n] = f32x4{0, 0, 0, 0};
      }
      for (; k0 < key_end; k0 += TILE) {
        load(s, k0, page);
        find(k0 + TILE, page);
        work(s, k0);
      }
      if (KIND == HERSCHEL_INT8 || apart) break;  // int8's codes are finite, what their scales make is a row's own
      float check = 0;                            // NaN if a sum is not finite
#pragma unroll
      for (int rb = 0; rb < RB; ++rb)
#pragma unroll
        for (int n = 0; n < ND; ++n)
#pragma unroll
          for (int i = 0; i < 4; ++i) check = __builtin_fmaf(o[rb][n][i], 0.0f, check);
      if (!__ballot(!(check == 0))) break;
      apart = true;  // from the reference that this pass ended with
      k0 = key_begin + wave * 32;
      if (k0 < key_end) find(k0, page);
    }

    // The four waves' parts of these rows, joined through LDS block by block.
    const bool whole = tile == 0 && n_tiles == tiles;
    if (tile == 0 && tid == 0)
      p.span[(int64_t)b * p.units + unit] =
          whole ? int2{-1, 0} : int2{2 * (int)blockIdx.x + (pos == begin ? 0 : 1), (int)share_of(pos + tiles - 1, U, G)};
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
          const float by = factor(all[w * WS + D], top);
          den += all[w * WS + D + 1] * by;
          if (by != 0) {
#pragma unroll
            for (int n = 0; n < ND; ++n) acc[n] += all[w * WS + d0 + n] * by;
          } else {
#pragma unroll
            for (int n = 0; n < ND; ++n) acc[n] += weighted(all[w * WS + d0 + n], by);
          }
        }
        if (whole) {
          const float inv = den > 0 ? 1.0f / den : den == 0 ? 0.0f : den;  // no key seen: 0; NaN stays
          const int64_t at = ((int64_t)b * p.a.new_tokens + r / p.group) * p.a.q_heads + head * p.group + r % p.group;
          uint32_t* out = (uint32_t*)((uint16_t*)p.a.out + at * D + d0);
#pragma unroll
          for (int n = 0; n < ND; n += 2) out[n / 2] = pack2<TYPE>(acc[n] * inv, acc[n + 1] * inv);
          if (p.a.lse && tid % 16 == 0) p.a.lse[at] = log_sum(top, den);
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
// workgroup per row, 16 lanes across the dimensions, each sixteenth part to a
// group of them, the groups through LDS.
template <int TYPE, int D, int RB>
__global__ __launch_bounds__(256) void k_decode_join(DecodeArgs p) {
  constexpr int ND = D / 16;
  __shared__ float s_part[16][D + 2];
  const int r = blockIdx.x % p.rows, of = blockIdx.x / p.rows;
  const int b = of / p.c.n_heads, head = of % p.c.n_heads, unit = head * p.row_blocks + r / (RB * 16);
  const int2 span = p.span[(int64_t)b * p.units + unit];
  if (span.x < 0) return;
  const int first = span.x / 2, last = span.y;  // shares; a later share's part is its first
  const int lane = threadIdx.x % 16, group = threadIdx.x / 16;
  float top, den, acc[ND];
  // Sums that are not finite are joined again with infinities kept where a factor is 0.
  auto add = [&](const float* from, auto kept) INLINE {
    const float t = from[D], to = fmaxf(top, t);
    const float old = factor(top, to), by = factor(t, to);
    den = den * old + from[D + 1] * by;
#pragma unroll
    for (int n = 0; n < ND; ++n)
      if constexpr (kept) acc[n] = weighted(acc[n], old) + weighted(from[lane * ND + n], by);
      else acc[n] = acc[n] * old + from[lane * ND + n] * by;
    top = to;
  };
  auto finite = [&]() INLINE {
    float check = 0;
#pragma unroll
    for (int n = 0; n < ND; ++n) check = __builtin_fmaf(acc[n], 0.0f, check);
    return check == 0;
  };
  auto of_group = [&](auto kept) INLINE {
    top = FAR_BELOW, den = 0;
#pragma unroll
    for (int n = 0; n < ND; ++n) acc[n] = 0;
    for (int w = first + group; w <= last; w += 16) {
      const int64_t slot = w == first ? span.x : 2 * w;
      add(p.part + (slot * (RB * 16) + r % (RB * 16)) * (D + 2), kept);
    }
  };
  of_group(std::false_type());
  if (!finite()) of_group(std::true_type());
#pragma unroll
  for (int n = 0; n < ND; ++n) s_part[group][lane * ND + n] = acc[n];
  if (lane == 0) {
    s_part[group][D] = top;
    s_part[group][D + 1] = den;
  }
  __syncthreads();
  if (group) return;
  const float own_top = top, own_den = den;
  for (int i = 1; i < 16 && i <= last - first; ++i) add(s_part[i], std::false_type());
  if (!finite()) {
    top = own_top, den = own_den;
#pragma unroll
    for (int n = 0; n < ND; ++n) acc[n] = s_part[0][lane * ND + n];
    for (int i = 1; i < 16 && i <= last - first; ++i) add(s_part[i], std::true_type());
  }
  const float inv = den > 0 ? 1.0f / den : den == 0 ? 0.0f : den;
  const int64_t at = ((int64_t)b * p.a.new_tokens + r / p.group) * p.a.q_heads + head * p.group + r % p.group;
  uint32_t* out = (uint32_t*)((uint16_t*)p.a.out + at * D + lane * ND);
#pragma unroll
  for (int n = 0; n < ND; n += 2) out[n / 2] = pack2<TYPE>(acc[n] * inv, acc[n + 1] * inv);
  if (p.a.lse && lane == 0) p.a.lse[at] = log_sum(top, den);
}

template <int TYPE, int KIND, int D, int RB>
static int decode_launch(DecodeArgs& p) {
  const size_t pre = ((p.a.n_seqs + 1 + 3) & ~3) * 4;
  const int rc = launch(k_decode<TYPE, KIND, D, RB>, dim3(256 * shares_of_cu(KIND, RB, D)), dim3(256), pre + 4 * 16 * (D + 2) * 4,
                        p.a.hip_stream, p);
  if (rc != HERSCHEL_OK) return rc;
  return launch(k_decode_join<TYPE, D, RB>, dim3((unsigned)(p.a.n_seqs * p.c.n_heads * p.rows)), dim3(256), 0,
                p.a.hip_stream, p);
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
  const int rows = new_tokens * (q_heads / cache->n_heads), block = decode_rows(rows);
  *bytes = (size_t)2 * MAX_SHARES * block * (cache->head_dim + 2) * 4 +
           (size_t)n_seqs * cache->n_heads * ((rows + block - 1) / block) * sizeof(int2);
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
  p.q_vec = chunks_aligned(a.q, a.q_strides) && (a.q_seq_stride & 7) == 0;
  p.group = a.q_heads / cache->n_heads;
  p.rows = a.new_tokens * p.group;
  const int block = decode_rows(p.rows);
  p.row_blocks = (p.rows + block - 1) / block;
  p.units = cache->n_heads * p.row_blocks;
  p.part = (float*)a.workspace;
  p.span = (int2*)(p.part + (size_t)2 * MAX_SHARES * block * (cache->head_dim + 2));
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
