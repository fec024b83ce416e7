// Products of rows with 4-bit weights, one launch, or two where long columns are
// shared among workgroups.
//
// y[m][n] = sum_g s[n][g] (sum_{k in g} c[n][k] x[m][k] - z[n][g] sum_{k in g} x[m][k]).
// The codes enter the matrix cores as what they are, 0 to 15: as bytes they are
// whole numbers for int8 rows, and read as fp8 they are c 2^-9 exactly (0 to 7 as its
// subnormals, 8 to 15 as its first eight normals), which an instruction turns into a
// pair of 16-bit elements.  fp8 rows become half on the way, exactly: the matrix
// cores' own fp8 products hold their sums to 2^-15 to 2^-19 of the magnitudes' sum
// only, in 16 bits they are whole to 32.
// The group's sum of x, which the zero needs, comes from one more product with a
// constant operand; scale and zero meet the group's sums, not the weights.
// The bytes of the weights bound large calls of few rows: four rows by a gated
// 25600 x 5120 matrix, 72 MB, 16.2 us, 4.4 TB/s with the start of the kernel (65 MB that
// are only read take 15 to 16; with other weights each time, 600 MB in turn, so that no
// cache holds them, 20.1); small ones their first loads' latency (one row by 6144 x 4096
// 6.5 us), 64 rows vector instructions (int8 by 5120 x 25600 27.9 us with the join, with
// weights in turn 31.0: 26.6 and 4.2), prompts the copies of x (2048 rows by 6144 x 4096
// 152 us, 680 TFLOP/s).
#pragma once

#include "ops.hpp"

namespace hop {

struct ProductArgs {
  herschel_product_args a;
  herschel_weights4 w;
  int tiles_k, tiles_n;  // tiles of 128 columns, of 16 weight rows
  int half;      // gated: tiles of 16 rows from a row to the one it gates
  int turns, turns_log;  // of the waves in a phase, a power of two
  int buffers;   // for phases, 2 or more
  int chunked;   // rows of x are whole chunks of 16 bytes
  int splits, tiles_split;  // workgroups that share the columns of a tile of the product, tiles of columns of each
};

typedef u32x4 u32x4_any __attribute__((aligned(1)));
typedef int i32x4 __attribute__((ext_vector_type(4)));

// The 16-bit type that rows of a kind, other than int8, and their codes meet in.
template <int KIND> constexpr int HALF_OF = KIND == HERSCHEL_FP8 ? HERSCHEL_F16 : KIND;

template <int KIND> struct Sum { typedef f32x4 T; };
template <> struct Sum<HERSCHEL_INT8> { typedef i32x4 T; };
template <int KIND> struct Operand { typedef u32x4 T; };  // eight elements
template <> struct Operand<HERSCHEL_INT8> { typedef u32x2 T; };

// D += A B of 32 columns: A the weights, 16 rows, B sixteen rows of x.
template <int KIND>
__device__ __forceinline__ typename Sum<KIND>::T mma(typename Operand<KIND>::T a, typename Operand<KIND>::T b,
                                                     typename Sum<KIND>::T c) {
  if constexpr (KIND == HERSCHEL_INT8)
    return __builtin_amdgcn_mfma_i32_16x16x32_i8(__builtin_bit_cast(long, a), __builtin_bit_cast(long, b), c, 0, 0, 0);
  else return mfma16<HALF_OF<KIND>>(a, b, c);
}
// The products of a group's operands: N of A, STEPS times 32 columns each, with one
// B, added to d.  int8 rows have an instruction for 64 columns in the time of 32 (16
// cycles a SIMD).  A product waits for its own last one: the N take turns.
template <int KIND, int STEPS, int N>
__device__ __forceinline__ void mma_group(typename Sum<KIND>::T* d, const typename Operand<KIND>::T (*a)[STEPS],
                                          const typename Operand<KIND>::T* b) {
  if constexpr (KIND == HERSCHEL_INT8 && STEPS > 1) {
#pragma unroll
    for (int j = 0; j < STEPS; j += 2) {
      const i32x4 v = {(int)b[j][0], (int)b[j][1], (int)b[j + 1][0], (int)b[j + 1][1]};
#pragma unroll
      for (int t = 0; t < N; ++t)
        d[t] = __builtin_amdgcn_mfma_i32_16x16x64_i8(
            i32x4{(int)a[t][j][0], (int)a[t][j][1], (int)a[t][j + 1][0], (int)a[t][j + 1][1]}, v, d[t], 0, 0, 0);
    }
  } else {
#pragma unroll
    for (int j = 0; j < STEPS; ++j)
#pragma unroll
      for (int t = 0; t < N; ++t) d[t] = mma<KIND>(a[t][j], b[j], d[t]);
  }
}

// Eight fp8 as an operand.
template <int KIND>
__device__ __forceinline__ u32x4 of_fp8(uint32_t lo, uint32_t hi) {
  constexpr int TO = HALF_OF<KIND>;
  return u32x4{decode2<HERSCHEL_FP8, TO, false>(lo), decode2<HERSCHEL_FP8, TO, true>(lo),
               decode2<HERSCHEL_FP8, TO, false>(hi), decode2<HERSCHEL_FP8, TO, true>(hi)};
}
// A word's eight codes as an operand: byte b holds columns b and b + 4.
template <int KIND>
__device__ __forceinline__ typename Operand<KIND>::T unpack_codes(uint32_t w) {
  const uint32_t lo = w & 0x0f0f0f0fu, hi = (w >> 4) & 0x0f0f0f0fu;
  if constexpr (KIND == HERSCHEL_INT8) return u32x2{lo, hi};
  else return of_fp8<KIND>(lo, hi);
}
// Ones in the codes' unit, in every place.
template <int KIND>
__device__ __forceinline__ typename Operand<KIND>::T ones() {
  if constexpr (KIND == HERSCHEL_INT8) return u32x2{0x01010101u, 0x01010101u};
  else return of_fp8<KIND>(0x01010101u, 0x01010101u);
}

// The sizes of a kernel: up to ROWS rows of x and WN waves' NT tiles of 16 weight
// rows a workgroup, whose WK waves share the columns, 128 each in turn; a wave's
// weights are asked for U times 128 columns ahead, and COPY waves bring x.
// GROUPS: rows of 8 bits with a scale for each of the weights' groups.
constexpr int PHASE_ALIGN = 128;
template <int KIND_, bool GROUPS_, int GROUP_, int ROWS_, int NT_, int WN_, int WK_, int U_, int COPY_, int LDS_>
struct Shape {
  static constexpr int KIND = KIND_, GROUP = GROUP_, ROWS = ROWS_, NT = NT_, WN = WN_, WK = WK_, U = U_, COPY = COPY_, LDS = LDS_;
  static constexpr bool GROUPS = GROUPS_;
  static constexpr int MT = (ROWS + 15) / 16;
  static constexpr int PER = 128 / GROUP, STEPS = GROUP / 32, RUN = GROUP / 4;
  static constexpr int WAVES = WN * WK, THREADS = (WAVES + COPY) * WAVE;
  static constexpr int EACH = quantised(KIND) ? 16 : 8;   // elements of a chunk of 16 bytes
  static constexpr int CHUNKS = 128 / EACH;               // of 128 columns of a row
  static constexpr int LEAST = WK * CHUNKS < WAVE ? WAVE / (WK * CHUNKS) : 1;  // turns of a phase: a copy is of one row
  // LDS bytes of a phase, `turns` times 128 columns for each of WK waves, from one multiple of PHASE_ALIGN to another
  static __host__ __device__ constexpr int phase_bytes(int rows, int turns) {
    return (rows * WK * turns * (CHUNKS * 16 + (GROUPS ? PER * 4 : 0)) + PHASE_ALIGN - 1) & -PHASE_ALIGN;
  }
  static_assert((WK & (WK - 1)) == 0, "a row's chunks of a phase are counted by shifts");
};

// What a wave reads of the weights for 128 columns.
template <class S>
struct Columns {
  u32x4 code[S::NT];
  u32x4 scale[S::NT][S::PER];  // four rows' scales and zeros
};
template <class S>
__device__ __forceinline__ void load_columns(Columns<S>& c, const ProductArgs& p, const int* tile, int kt, int lane) {
#pragma unroll
  for (int t = 0; t < S::NT; ++t) {
    const int64_t at = (int64_t)kt * p.tiles_n + tile[t];
    c.code[t] = *((const u32x4*)p.w.codes + at * WAVE + lane);
#pragma unroll
    for (int g = 0; g < S::PER; ++g) c.scale[t][g] = *((const u32x4*)p.w.scales + (at * 4 + lane / 16) * S::PER + g);
  }
}

template <class T>
__device__ __forceinline__ T lds_at(uint32_t address) {
  return *(const __attribute__((address_space(3))) T*)(uintptr_t)address;
}

// Where a lane's part of a row of x begins in a phase in LDS: a row's chunks lie in
// order but for the lowest three bits of their number, which the row's turn, so
// that sixteen rows' reads of one chunk meet every bank equally often.  The bits of the
// rest of a column are apart from all these, and a phase and 128 columns of it
// begin at multiples of 128 bytes (the scales behind a phase's rows fill it up to one:
// those of an odd number of rows in groups of 64 end in the middle).
template <class S>
__device__ __forceinline__ uint32_t lane_part(int row, int row_bytes, int lane) {
  return row * row_bytes + ((lane / 16 * S::RUN * (16 / S::EACH)) ^ ((row & 7) * 16));
}

// 128 columns: the sums of each tile of rows and of weight rows, x and its scales from LDS.
template <class S>
__device__ __forceinline__ void add_columns(f32x4 (*sum)[S::NT], const Columns<S>& c, const uint32_t* part, uint32_t at,
                                            const uint32_t* scale_part, uint32_t scale_at) {
  constexpr int KIND = S::KIND, STEPS = S::STEPS, NT = S::NT;
  typedef typename Operand<KIND>::T Op;
#pragma unroll
  for (int g = 0; g < S::PER; ++g) {
    Op codes[NT + 1][STEPS];
    float s[NT][4], z[NT][4];
#pragma unroll
    for (int j = 0; j < STEPS; ++j) codes[NT][j] = ones<KIND>();
#pragma unroll
    for (int t = 0; t < NT; ++t) {
#pragma unroll
      for (int j = 0; j < STEPS; ++j) codes[t][j] = unpack_codes<KIND>(c.code[t][g * STEPS + j]);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        s[t][e] = __builtin_bit_cast(float, c.scale[t][g][e] & 0xffffff00u);
        z[t][e] = (float)(c.scale[t][g][e] & 0xffu);
      }
    }
#pragma unroll
    for (int i = 0; i < S::MT; ++i) {
      const uint32_t from = at + part[i];
      Op b[STEPS];
#pragma unroll
      for (int j = 0; j < STEPS; ++j) {
        const uint32_t here = from ^ ((g * S::GROUP + j * 8) * (16 / S::EACH));
        if constexpr (KIND == HERSCHEL_FP8) {
          const u32x2 w = lds_at<u32x2>(here);
          b[j] = of_fp8<KIND>(w[0], w[1]);
        } else {
          b[j] = lds_at<Op>(here);
        }
      }
      float by = 1.0f;
      if constexpr (S::GROUPS) by = lds_at<float>(scale_at + scale_part[i] + g * 4);
      typename Sum<KIND>::T d[NT + 1];
#pragma unroll
      for (int t = 0; t <= NT; ++t) d[t] = typename Sum<KIND>::T{0, 0, 0, 0};
      mma_group<KIND, STEPS, NT + 1>(d, codes, b);
      const float of_x = (float)d[NT][0];  // the sum of the lane's row of x, in the codes' unit
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          float y = (float)d[t][e] - z[t][e] * of_x;
          if (S::GROUPS) y *= by;
          sum[i][t][e] += y * s[t][e];
        }
      // The sums are taken here: left alone, the compiler keeps the products of several turns and adds them later,
      // which takes more registers than there are.
#pragma unroll
      for (int t = 0; t < NT; ++t) asm volatile("" : "+v"(sum[i][t]));
    }
  }
}

// Waits until no more than n of the wave's copies are under way, or fewer.
__device__ __forceinline__ void wait_copies(int n) {
  if (n >= 32) __builtin_amdgcn_s_waitcnt(0x8070);       // vmcnt 32, lgkmcnt 0
  else if (n >= 16) __builtin_amdgcn_s_waitcnt(0x4070);
  else if (n >= 8) __builtin_amdgcn_s_waitcnt(0x0078);
  else if (n >= 4) __builtin_amdgcn_s_waitcnt(0x0074);
  else if (n >= 2) __builtin_amdgcn_s_waitcnt(0x0072);
  else if (n >= 1) __builtin_amdgcn_s_waitcnt(0x0071);
  else __builtin_amdgcn_s_waitcnt(0x0070);
}

// The copying waves' part of a phase: its columns of x, from tile0 on, to LDS.  Whole phases of rows
// of whole chunks go there directly.
template <class S>
__device__ __forceinline__ void copy_phase(const ProductArgs& p, char* to, int64_t m0, int rows, int tile0, int copier, int lane) {
  const herschel_product_args& a = p.a;
  constexpr int BYTES = 16 / S::EACH;
  const int K = p.w.k, k0 = tile0 * 128;
  const int shift = p.turns_log + __builtin_ctz(S::WK * S::CHUNKS), size = rows << shift, mask = (1 << shift) - 1;
  if (p.chunked && k0 + S::WK * p.turns * 128 <= K) {
    const int64_t step = S::COPY * a.x_row * BYTES;
    for (int at = 0; at <= mask; at += WAVE) {  // a copy is of one row
      const char* from = (const char*)a.x + ((m0 + copier) * a.x_row + k0) * BYTES + at * 16;
      for (int r = copier; r < rows; r += S::COPY, from += step)
        copy_to_lds(from + ((lane ^ (r & 7)) * 16), to + ((r << shift) + at) * 16);
    }
  } else {
#pragma unroll 4
    for (int id = copier * WAVE + lane; id < size; id += S::COPY * WAVE) {
      const int r = id >> shift, k = k0 + (id & mask) * S::EACH;
      const char* row = (const char*)a.x + (m0 + r) * a.x_row * BYTES;
      if (k + S::EACH <= K) *(u32x4*)(to + (id ^ (r & 7)) * 16) = *(const u32x4_any*)(row + (int64_t)k * BYTES);
      else if (k >= K) *(u32x4*)(to + (id ^ (r & 7)) * 16) = u32x4{0, 0, 0, 0};
    }
    const int odd = K % S::EACH, k = K - odd;  // a row's last elements, where they fill no chunk
    if (odd && k >= k0 && k < k0 + S::WK * p.turns * 128) {
      for (int r = copier * WAVE + lane; r < rows; r += S::COPY * WAVE) {
        const char* from = (const char*)a.x + ((m0 + r) * a.x_row + k) * BYTES;
        u32x4 w = {0, 0, 0, 0};
#pragma unroll
        for (int e = 0; e < S::EACH; ++e) {
          const uint32_t v = e >= odd ? 0u : BYTES == 1 ? *(const uint8_t*)(from + e) : *(const uint16_t*)(from + 2 * e);
          w[e * BYTES / 4] |= v << (8 * BYTES * (e % (4 / BYTES)));
        }
        *(u32x4*)(to + (((r << shift) + (k - k0) / S::EACH) ^ (r & 7)) * 16) = w;
      }
    }
    // Said here, so that the compiler does not wait in the loop above for registers that these loads may have left
    // under way: before every copy, 65 us where 26 are enough (16 rows by 5120 x 25600 weights).
    __builtin_amdgcn_s_waitcnt(0x0070);
  }
  if constexpr (S::GROUPS) {
    const int groups = (K + S::GROUP - 1) / S::GROUP, each = S::WK * S::PER * p.turns;
    for (int id = copier * WAVE + lane; id < rows * each; id += S::COPY * WAVE) {
      const int r = id / each, g = tile0 * S::PER + id % each;
      *(float*)(to + size * 16 + id * 4) = a.x_scale[(m0 + r) * groups + min(g, groups - 1)];
    }
  }
}

// Four elements of the product's row m from column n on, from their sums (gated: y's gate b).
__device__ __forceinline__ void store_product(const herschel_product_args& a, const herschel_weights4& w, int kind, bool groups,
                                              int64_t m, int n, f32x4 y, f32x4 b) {
  const int n_out = a.gated ? w.n / 2 : w.n;
  if (n >= n_out) return;
  float by = kind == HERSCHEL_INT8 ? 1.0f : 512.0f;
  if (quantised(kind) && !groups) by *= a.x_scale[m];
  y *= by;
  if (a.gated) {
    b *= by;
#pragma unroll
    for (int e = 0; e < 4; ++e) y[e] = y[e] / (1.0f + expf(-y[e])) * b[e];
  }
  const bool bf = a.type == HERSCHEL_BF16;
  const uint32_t w0 = bf ? pack2<HERSCHEL_BF16>(y[0], y[1]) : pack2<HERSCHEL_F16>(y[0], y[1]);
  const uint32_t w1 = bf ? pack2<HERSCHEL_BF16>(y[2], y[3]) : pack2<HERSCHEL_F16>(y[2], y[3]);
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

// A workgroup takes the tiles that its shape says (gated: half of a wave's of the
// rows that gate, half of those that they gate).  x comes through LDS in phases, up
// to six in turn, which waves of their own bring: loads are waited for in their order, and
// x's between those of weights asked for long before would have these waited for too.
// The weights go straight to registers, in no branch, so that the count of
// what may still be under way is known.  The waves' sums meet in LDS.
template <class S>
__global__ __launch_bounds__(S::THREADS) void k_product4(ProductArgs p) {
  constexpr int KIND = S::KIND, MT = S::MT, NT = S::NT, U = S::U, WK = S::WK;
  const herschel_product_args& a = p.a;
  const herschel_weights4& w = p.w;
  extern __shared__ __attribute__((aligned(PHASE_ALIGN))) f32x4 parts[];
  const int lane = threadIdx.x % WAVE, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / WAVE), wk = wave % WK, wn = wave / WK;
  const int64_t m0 = (int64_t)blockIdx.y * S::ROWS;
  const int rows = (int)min((int64_t)S::ROWS, a.n_rows - m0);
  const bool gated = a.gated != 0;
  const int last_n = gated ? p.half : (w.n + 15) / 16, outs = gated ? NT / 2 : NT;
  const int bytes = S::phase_bytes(rows, p.turns), tile0 = (int)blockIdx.z * p.tiles_split;
  const int tiles = min(p.tiles_split, p.tiles_k - tile0), turns_all = (tiles + WK - 1) / WK;
  // The workgroup's waves meet: x of a phase is there, and the phase before has been used.
  auto meet = [] {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0xc07f);  // lgkmcnt 0
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
  };

  if (wave >= S::WAVES) {
    // BUFFERS - 1 phases are under way or in use.  A wave's copies end in their order.
    const int phases = (turns_all + p.turns - 1) >> p.turns_log, copier = wave - S::WAVES;
    const int copies = (rows + S::COPY - 1 - copier) / S::COPY * (S::WK * p.turns * S::CHUNKS / WAVE);  // of a phase
    for (int phase = 0; phase < p.buffers - 1 && phase < phases; ++phase)
      copy_phase<S>(p, (char*)parts + phase * bytes, m0, rows, tile0 + (phase * WK << p.turns_log), copier, lane);
    int to = p.buffers - 1;
    for (int phase = 0; phase <= phases; ++phase) {
      asm volatile("" ::: "memory");
      const int ahead = min(p.buffers - 2, phases - 1 - phase);  // the last phase may have copies of another number
      wait_copies(ahead > 0 && phase + ahead < phases - 1 ? ahead * copies : ahead > 0 ? (ahead - 1) * copies : 0);
      meet();
      if (phase + p.buffers - 1 < phases)
        copy_phase<S>(p, (char*)parts + to * bytes, m0, rows, tile0 + ((phase + p.buffers - 1) * WK << p.turns_log), copier, lane);
      to = to + 1 == p.buffers ? 0 : to + 1;
    }
  } else {
    const int first = ((int)blockIdx.x * S::WN + wn) * outs;
    int tile[NT];  // tiles beyond the last are computed as it and not stored
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      if (gated) tile[t] = min(first + t % (NT > 1 ? NT / 2 : 1), last_n - 1) + (t >= NT / 2 ? p.half : 0);
      else tile[t] = min(first + t, last_n - 1);
    }
    f32x4 sum[MT][NT];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
      for (int t = 0; t < NT; ++t) sum[i][t] = f32x4{0, 0, 0, 0};
    Columns<S> c[U];
#pragma unroll
    for (int u = 0; u < U; ++u) load_columns(c[u], p, tile, tile0 + min(u * WK + wk, tiles - 1), lane);
    // the phase's x, and where a lane's parts of its rows are in it; rows beyond the last are computed as it and not stored
    const uint32_t begin = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)(char*)parts, end = begin + p.buffers * bytes;
    const int of = WK << p.turns_log;
    uint32_t from = begin, part[MT], scale_part[MT];
#pragma unroll
    for (int i = 0; i < MT; ++i) {
      const int r = min(16 * i + lane % 16, rows - 1);
      part[i] = lane_part<S>(r, of * (S::CHUNKS * 16), lane);
      scale_part[i] = (rows * S::CHUNKS * 16 + r * S::PER * 4) * of;
    }
    auto next = [&] {
      meet();
      from += bytes;
      if (from == end) from = begin;
    };
    // turn n of the waves
    auto work = [&](int n, const Columns<S>& c) {
      const int at = (n & (p.turns - 1)) * WK + wk;
      add_columns<S>(sum, c, part, from + at * (S::CHUNKS * 16), scale_part, from + at * (S::PER * 4));
    };
    meet();
    int n = 0;
    for (; n + U < turns_all; n += U) {
#pragma unroll
      for (int u = 0; u < U; ++u) {
        work(n + u, c[u]);
        load_columns(c[u], p, tile, tile0 + min((n + u + U) * WK + wk, tiles - 1), lane);
        if (((n + u + 1) & (p.turns - 1)) == 0) next();
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (n + u >= turns_all) break;
      if ((n + u) * WK + wk < tiles) work(n + u, c[u]);
      if (((n + u + 1) & (p.turns - 1)) == 0 || n + u + 1 == turns_all) next();
    }
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
      for (int t = 0; t < NT; ++t) parts[((wave * MT + i) * NT + t) * WAVE + lane] = sum[i][t];
  }
  __syncthreads();
  for (int o = threadIdx.x; o < S::WN * MT * outs * WAVE; o += S::THREADS) {
    const int l = o % WAVE, t = o / WAVE % outs, v = o / WAVE / outs % S::WN, i = o / WAVE / outs / S::WN;
    const int64_t m = m0 + 16 * i + l % 16;
    const int at = ((int)blockIdx.x * S::WN + v) * outs + t;
    if (m >= m0 + rows || at >= last_n) continue;
    f32x4 y = {0, 0, 0, 0}, b = {0, 0, 0, 0};
#pragma unroll
    for (int k = 0; k < WK; ++k) {
      y += parts[(((v * WK + k) * MT + i) * NT + t) * WAVE + l];
      if (gated) b += parts[(((v * WK + k) * MT + i) * NT + t + outs) * WAVE + l];
    }
    const int n = 16 * at + 4 * (l / 16);
    if (p.splits == 1) {
      store_product(a, w, KIND, S::GROUPS, m, n, y, b);
    } else {
      float* to = (float*)a.workspace + ((int64_t)blockIdx.z * a.n_rows + m) * (p.tiles_n * 16);
      *(f32x4*)(to + n) = y;
      if (gated) *(f32x4*)(to + p.half * 16 + n) = b;
    }
  }
}

// The sums of the workgroups that share a product's columns, four of its elements a thread.
template <bool GROUPS>
__global__ __launch_bounds__(256) void k_product4_join(ProductArgs p) {
  const int64_t m = blockIdx.y;
  const int n = (int)(blockIdx.x * 256 + threadIdx.x) * 4;
  if (n >= p.tiles_n * 16 / (p.a.gated ? 2 : 1)) return;
  const float* from = (const float*)p.a.workspace + m * (p.tiles_n * 16) + n;
  f32x4 y = {0, 0, 0, 0}, b = {0, 0, 0, 0};
  f32x4 part[4], gate_part[4];
#pragma unroll
  for (int z = 0; z < 4; ++z) {  // all asked for before the first is used
    part[z] = gate_part[z] = f32x4{0, 0, 0, 0};
    if (z < p.splits) part[z] = *(const f32x4*)from;
    if (z < p.splits && p.a.gated) gate_part[z] = *(const f32x4*)(from + p.half * 16);
    from += p.a.n_rows * (p.tiles_n * 16);
  }
#pragma unroll
  for (int z = 0; z < 4; ++z) y += part[z], b += gate_part[z];
  store_product(p.a, p.w, p.a.kind, GROUPS, m, n, y, b);
}

template <class S>
static int product_launch(ProductArgs& p, int splits) {  // at most 4
  static_assert(2 * S::phase_bytes(S::ROWS, S::LEAST) <= S::LDS, "two phases must fit");
  const int tiles = p.a.gated ? p.half : p.tiles_n, each = S::WN * (p.a.gated ? S::NT / 2 : S::NT);
  const int64_t blocks = (p.a.n_rows + S::ROWS - 1) / S::ROWS;  // at most 65535
  p.tiles_split = (p.tiles_k + splits - 1) / splits;
  p.splits = (p.tiles_k + p.tiles_split - 1) / p.tiles_split;
  const int rows = p.a.n_rows < S::ROWS ? (int)p.a.n_rows : S::ROWS, turns_all = (p.tiles_split + S::WK - 1) / S::WK;
  constexpr int BYTES = 16 / S::EACH;
  p.chunked = p.w.k % S::EACH == 0 && aligned(p.a.x, 16) && p.a.x_row * BYTES % 16 == 0;
  p.turns = S::LEAST;
  while (p.turns < turns_all && 4 * S::phase_bytes(rows, 2 * p.turns) <= S::LDS) p.turns *= 2;
  p.turns_log = log2i(p.turns);
  const int phases = (turns_all + p.turns - 1) / p.turns, fit = S::LDS / S::phase_bytes(rows, p.turns);
  p.buffers = phases < 2 ? 2 : phases < fit ? phases : fit;
  if (p.buffers > 6) p.buffers = 6;
  size_t lds = (size_t)p.buffers * S::phase_bytes(rows, p.turns);
  const size_t sums = (size_t)S::WAVES * S::MT * S::NT * WAVE * sizeof(f32x4);
  if (lds < sums) lds = sums;
  const int code = launch(k_product4<S>, dim3((unsigned)((tiles + each - 1) / each), (unsigned)blocks, (unsigned)p.splits),
                          dim3(S::THREADS), lds, p.a.hip_stream, p);
  if (code != HERSCHEL_OK || p.splits == 1) return code;
  return launch(S::GROUPS ? k_product4_join<true> : k_product4_join<false>,
                dim3((unsigned)((tiles * 4 + 255) / 256), (unsigned)p.a.n_rows), dim3(256), 0, p.a.hip_stream, p);
}
// Which kernel a call takes.  A workgroup's start and end cost as much as several
// turns, so that one round of workgroups, at most one a CU, is best: with few weight
// rows narrow ones, with many wide ones; with few weight rows and long columns these
// are shared among several, joined by a second kernel.  The time of each choice
// is estimated from measured ones (bf16 rows, groups of 128; two thirds for many int8 rows), in units of 10 ns: 400
// and so much a turn, 600 for the join and its launch.  Measured against the choices beside them: 16
// rows by 25600 x 5120 weights 17.3 us with 8 tiles a workgroup, 21.2 with 4, 29.5
// with 2; by 6144 x 4096 7.9 with 2, 9.5 with 4, 11.6 with 1; by 1280 x 5120 7.2 with 1, 8.4 with 2; by 5120 x 25600 22.8 with 4 in three parts,
// 26.4 with 2 and no parts; by 4096 x 14336 13.8 with 2 in two parts, 16.3 without.
// fp8 rows and groups of 32 and 64 go by the same times: the choices beside theirs have
// not been measured.
struct Choice {
  int wide;    // 0 to 3: one, two, four, eight tiles of weight rows a workgroup
  int splits;
};
inline size_t parts_bytes(const ProductArgs& p, int splits) { return (size_t)splits * p.a.n_rows * p.tiles_n * 64; }
inline int rows_at_once(int64_t n_rows) { return n_rows <= 16 ? 16 : n_rows <= 32 ? 32 : 64; }
constexpr int64_t MOST_SHARED = 4096;  // rows whose columns are shared: more fill the card without, and are too many to join
inline Choice choose(const ProductArgs& p, size_t room) {
  if (p.a.n_rows > MOST_SHARED) room = 0;
  static const int TURN[3][4] = {{65, 95, 75, 65}, {0, 175, 105, 85}, {0, 156, 190, 135}}, WAVES_K[2][4] = {{8, 8, 4, 2}, {0, 4, 4, 2}};
  const int rows = rows_at_once(p.a.n_rows), rows_at = rows / 32;
  // a wave with one tile of weight rows has none that gates
  const int narrowest = rows == 16 && !p.a.gated ? 0 : rows == 64 && p.a.gated ? 2 : 1;
  const int64_t tiles = p.a.gated ? p.half * 2 : p.tiles_n, blocks_m = (p.a.n_rows + rows - 1) / rows;
  Choice best{narrowest, 1};
  int64_t least = INT64_MAX;
  for (int wide = narrowest; wide < 4; ++wide) {
    const int64_t blocks = (tiles + (1 << wide) - 1) / (1 << wide) * blocks_m;
    for (int splits = 1; splits <= 4; ++splits) {
      if (splits > 1 && parts_bytes(p, splits) > room) break;
      const int each = (p.tiles_k + splits - 1) / splits, k = WAVES_K[rows == 64][wide];
      const int64_t rounds = (blocks * splits + 255) / 256, turns = (each + k - 1) / k;
      const int turn = p.a.kind == HERSCHEL_INT8 && rows > 16 ? TURN[rows_at][wide] * 2 / 3 : TURN[rows_at][wide];
      const int64_t time = rounds * (400 + turns * turn) + (splits > 1 ? 600 : 0);
      if (time < least) {
        least = time;
        best = Choice{wide, splits};
      }
    }
  }
  return best;
}

template <int KIND, bool GROUPS, int GROUP>
static int product_shape(ProductArgs& p) {
  constexpr int U = GROUP == 32 ? 1 : 2;  // more groups' scales of more turns ahead do not fit the registers
  const int rows = rows_at_once(p.a.n_rows);
  const size_t room = p.a.workspace && aligned(p.a.workspace, 16) ? p.a.workspace_bytes : 0;
  const Choice c = choose(p, room);
  if (rows == 16) {
    if (c.wide == 0) return product_launch<Shape<KIND, GROUPS, GROUP, 16, 1, 1, 8, 2 * U, 4, 131072>>(p, c.splits);
    if (c.wide == 1) return product_launch<Shape<KIND, GROUPS, GROUP, 16, 2, 1, 8, U, 4, 131072>>(p, c.splits);
    if (c.wide == 2) return product_launch<Shape<KIND, GROUPS, GROUP, 16, 2, 2, 4, U, 4, 131072>>(p, c.splits);
    return product_launch<Shape<KIND, GROUPS, GROUP, 16, 2, 4, 2, U, 4, 131072>>(p, c.splits);
  }
  if (rows == 32) {
    if (c.wide == 1) return product_launch<Shape<KIND, GROUPS, GROUP, 32, 2, 1, 8, U, 4, 147456>>(p, c.splits);
    if (c.wide == 2) return product_launch<Shape<KIND, GROUPS, GROUP, 32, 2, 2, 4, U, 4, 131072>>(p, c.splits);
    return product_launch<Shape<KIND, GROUPS, GROUP, 32, 2, 4, 2, U, 4, 131072>>(p, c.splits);
  }
  if (c.wide == 1) return product_launch<Shape<KIND, GROUPS, GROUP, 64, 1, 2, 4, U, 4, 147456>>(p, c.splits);
  if (c.wide == 2) return product_launch<Shape<KIND, GROUPS, GROUP, 64, 2, 2, 4, U, 4, 147456>>(p, c.splits);
  return product_launch<Shape<KIND, GROUPS, GROUP, 64, 2, 4, 2, U, 4, 147456>>(p, c.splits);
}
template <int KIND, bool GROUPS>
static int product_group(ProductArgs& p) {
  switch (p.w.group) {
    case 32: return product_shape<KIND, GROUPS, 32>(p);
    case 64: return product_shape<KIND, GROUPS, 64>(p);
    default: return product_shape<KIND, GROUPS, 128>(p);
  }
}

// One of these for each kind of rows, in files of their own: they take long to compile.
int product_bf16(ProductArgs& p);
int product_f16(ProductArgs& p);
int product_fp8(ProductArgs& p);
int product_fp8_groups(ProductArgs& p);
int product_int8(ProductArgs& p);
int product_int8_groups(ProductArgs& p);

}  // namespace hop
