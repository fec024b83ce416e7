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
//  - A wave has 32 rows and two waves share a SIMD: one wave alone issues a VALU
//    instruction every 6 cycles, two every 3, and the exponentials of one run
//    beside the products of the other.  Eight waves in one workgroup take turns,
//    half of them at the products while the other half is at the exponentials;
//    with four, two workgroups of a CU drift apart by themselves.
//  - Keys and values go to LDS by rows without passing registers, the next tile
//    of values and the next two of keys while this one is worked on.  The chunks
//    of a row are permuted by the row's number, differently for K and V, which
//    spreads a wave's reads over all banks.  V's operand has its keys in a lane:
//    reads that transpose blocks of four keys by 16 dimensions deliver it.
//  - The reference of a row's exponentials stays as long as a tile's sum shows
//    that it fits (ops.hpp); else the maximum is taken and the accumulators
//    scaled.  No maximum is computed otherwise.
//  - Only tiles in which some row does not see some key are masked.  A hidden
//    key's exponential is 0, which an infinite or NaN value turns into NaN: a
//    wave whose sums are not finite at the end computes its rows again, with
//    nothing but the keys that each row sees.
//
// 32 heads of 128, causal, bf16, by the card: 4096 rows 141 to 146 us, 940 to 976
// TFLOP/s; three prompts of 2001 to 8192 rows 675 to 702 us, 1021 to 1061 TFLOP/s,
// where a matrix product of 8192 cubed reaches 1173 to 1201.
#include <algorithm>
#include <type_traits>

#include "ops.hpp"

namespace hop {

constexpr int KT = 64;      // keys of a tile
constexpr float NO_KEY = -3.0e38f;

#define INLINE __attribute__((always_inline))

struct PromptArgs {
  herschel_prompt_args a;
  int group;
  int levels;  // query tiles of the longest sequence
  int spread;  // XCDs that share a key head's workgroups; 0: heads in turn
  int splits;  // parts of each workgroup's keys (gridDim.y); above 1 they meet in k_prompt_join
  int packed;  // few rows: workgroups are numbered by the levels that the sequences have, not levels by sequences
};

// The rows and level (of 32) of workgroup `id` of packed ones: sequence after
// sequence, each from its last level (the longest) down; false beyond the last.
// Starts that fall count as the largest before them, so that the levels never
// exceed the rows' and one for each sequence.
__device__ __forceinline__ bool find_level(const herschel_prompt_args& a, int heads, uint32_t id, int& b, int& level, int64_t& q0,
                                           int64_t& q1) {
  const int lane = threadIdx.x % WAVE;
  auto at = [](int x, int l) INLINE { return __builtin_amdgcn_readlane(x, l); };
  int past = 0;
  for (int b0 = 0; b0 < a.n_seqs; b0 += WAVE) {
    int lo = (int)min((int64_t)max(a.cu_q[min(b0 + lane, a.n_seqs)], 0), a.n_q);
    int hi = (int)min((int64_t)max(a.cu_q[min(b0 + lane + 1, a.n_seqs)], 0), a.n_q);
    if (__ballot(hi < lo || lo < past)) {
      lo = max(lo, past);
#pragma unroll
      for (int o = 1; o < WAVE; o *= 2) lo = max(lo, __shfl_up(lo, o));  // the first lanes get their own
      hi = max(hi, lo);
    }
    const int n = (int)(((int64_t)min(hi - lo, a.max_q) * heads + 31) / 32);
    int sum = n;
#pragma unroll
    for (int o = 1; o < WAVE; o *= 2) {
      const int y = __shfl_up(sum, o);
      if (lane >= o) sum += y;
    }
    const uint64_t reached = __ballot((uint32_t)sum > id);
    if (reached) {
      const int l = __builtin_ctzll(reached);
      b = b0 + l;
      level = at(sum, l) - 1 - (int)id;
      q0 = at(lo, l);
      q1 = at(hi, l);
      return true;
    }
    id -= (uint32_t)at(sum, WAVE - 1);
    past = at(hi, WAVE - 1);
  }
  return false;
}

// What the workgroups of single sequences report where there may be none: the first wave of the grid.
__device__ __forceinline__ void report_lengths(const herschel_prompt_args& a) {
  for (int b = threadIdx.x; b < a.n_seqs; b += WAVE) {
    const int64_t q0 = a.cu_q[b], q1 = a.cu_q[b + 1], k0 = a.cu_k[b], k1 = a.cu_k[b + 1];
    if (q0 < 0 || (b == 0 && q0 > 0) || q1 < q0 || q1 > a.n_q || q1 - q0 > a.max_q || k0 < 0 || k1 < k0 || k1 > a.n_k) flag(a.status, HERSCHEL_OP_BAD_LENGTH);
  }
}

// Outputs [from, to) of heads h0 ... h0 + heads - 1 that no query computes: 0, log sums minus infinity.  The work of
// workgroup `id` of `of`.
template <int D>
__device__ __forceinline__ void no_query(const herschel_prompt_args& a, int64_t from, int64_t to, int h0, int heads, int64_t id,
                                         int64_t of) {
  const int chunks = heads * (D / 4);  // of 8 bytes, in a row
  for (int64_t x = id * blockDim.x + threadIdx.x; x < (to - from) * chunks; x += of * blockDim.x) {
    const int64_t at = (from + x / chunks) * a.q_heads + h0;
    ((u32x2*)((uint16_t*)a.out + at * D))[x % chunks] = u32x2{0, 0};
    if (a.lse && x % chunks < heads) a.lse[at + x % chunks] = -INFINITY;
  }
}
// The smallest and the largest start of a sequence, within the rows: what lies outside is no sequence's, and from the
// first start to the largest every row is one's.
__device__ __forceinline__ void start_range(const herschel_prompt_args& a, int64_t& lo, int64_t& hi) {
  lo = a.n_q, hi = 0;
  for (int b = threadIdx.x % WAVE; b <= a.n_seqs; b += WAVE) {
    const int64_t x = min(max((int64_t)a.cu_q[b], (int64_t)0), a.n_q);
    lo = min(lo, x), hi = max(hi, x);
  }
#pragma unroll
  for (int o = 1; o < WAVE; o *= 2) {
    lo = min(lo, (int64_t)__shfl_xor((int)lo, o));
    hi = max(hi, (int64_t)__shfl_xor((int)hi, o));
  }
}
// Rows without a query: beyond max_q of sequence b ([q0 + nq, q1)), before the first sequence and after the last;
// q0w and q1w are the sequence's starts as given.
template <int D>
__device__ __forceinline__ void rows_without(const herschel_prompt_args& a, int b, int64_t q0w, int64_t q1w, int64_t q0, int64_t q1,
                                             int nq, int h0, int heads, int id, int of) {
  if (q1 - q0 > nq) no_query<D>(a, q0 + nq, q1, h0, heads, id, of);
  const bool before = b == 0 && q0w > 0, after = b == a.n_seqs - 1 && q1w < a.n_q;
  if (before || after) {
    int64_t lo, hi;
    start_range(a, lo, hi);
    if (before) no_query<D>(a, 0, lo, h0, heads, id, of);
    for (int64_t row = lo + id; before && row < q0; row += of) {  // starts fall below the first: is the row one's?
      uint64_t named = 0;
      for (int s0 = 0; s0 < a.n_seqs && !named; s0 += WAVE) {
        const int s = s0 + threadIdx.x % WAVE;
        named = __ballot(s < a.n_seqs && a.cu_q[min(s, a.n_seqs - 1)] <= row && row < a.cu_q[min(s, a.n_seqs - 1) + 1]);
      }
      if (!named) no_query<D>(a, row, row + 1, h0, heads, 0, 1);
    }
    if (after) no_query<D>(a, hi, a.n_q, h0, heads, id, of);
  }
}

// A row's part: sums of its values, reference and sum of its exponentials.
template <int D>
constexpr int PART_FLOATS = D + 4;
template <int D>
__device__ __forceinline__ float* row_part(const herschel_prompt_args& a, int part, int64_t at) {
  return (float*)a.workspace + (part * (a.n_q * a.q_heads) + at) * PART_FLOATS<D>;
}

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4 LdsHalves;

// A wave's copy of 64 chunks of 16 bytes from global memory to consecutive LDS.
__device__ __forceinline__ void copy_to_lds(const void* from, void* to) {
  __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)from,
                                   (__attribute__((address_space(3))) void*)to, 16, 0, 0);
}

// Orders N products and their READS LDS reads each: AHEAD products' reads
// first, then one product and the reads of a later one in turn.  Left alone, the
// compiler waits for each read just before its product: 60 cycles of 32.
constexpr int AHEAD = 4;
template <int N, int READS, int GROUP>
__device__ __forceinline__ void reads_ahead() {
  __builtin_amdgcn_sched_group_barrier(0x100, AHEAD * READS, GROUP);
#pragma unroll
  for (int i = 0; i < N - AHEAD; ++i) {
    __builtin_amdgcn_sched_group_barrier(0x008, 1, GROUP);
    __builtin_amdgcn_sched_group_barrier(0x100, READS, GROUP);
  }
  __builtin_amdgcn_sched_group_barrier(0x008, AHEAD, GROUP);
}

// A row's outputs from the keys [lo, hi) alone, by a wave: 64 keys at a time, a
// key to a lane for the scores, then a dimension (or two) to a lane for the
// values, 32 rows asked for at once.  An infinite value or sum stays one, also
// where its weight is too small for 32 bits.  4096 rows of 32 heads of 128 that all see a NaN: 15 ms (a key at a time 46).
template <int TYPE, int D>
__device__ __forceinline__ void row_by_key(const uint16_t* q, const uint16_t* kbase, const uint16_t* vbase,
                                           const herschel_prompt_args& a, int lo, int hi, int64_t at) {
  constexpr int ND = D / WAVE, AT_ONCE = 32;
  const int lane = threadIdx.x % WAVE;
  lo = __builtin_amdgcn_readfirstlane(lo);
  hi = __builtin_amdgcn_readfirstlane(hi);
  const bool vec = ((uintptr_t)kbase & 15) == 0 && (a.k_strides.row & 7) == 0;
  float qv[ND], acc[ND], top = NO_KEY, den = 0, unused;
#pragma unroll
  for (int d = 0; d < ND; ++d) {
    unpack2<TYPE>(q[d * WAVE + lane], qv[d], unused);
    acc[d] = 0;
  }
  auto of_lane = [](float x, int i) INLINE {
    return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, x), i));
  };
  for (int k0 = lo; k0 < hi; k0 += WAVE) {
    const int n = min(WAVE, hi - k0);
    const uint16_t* k = kbase + (k0 + min(lane, n - 1)) * a.k_strides.row;
    float x = 0;
#pragma unroll
    for (int d0 = 0; d0 < D; d0 += 64) {
      u32x4 w[8];
      if (vec) {
#pragma unroll
        for (int c = 0; c < 8; ++c) w[c] = *(const u32x4*)(k + d0 + 8 * c);
      } else {
#pragma unroll
        for (int c = 0; c < 8; ++c) w[c] = load_elements(k + d0 + 8 * c);
      }
#pragma unroll
      for (int i = 0; i < 32; ++i) {
        float ka, kb;
        unpack2<TYPE>(w[i / 4][i % 4], ka, kb);
        x += of_lane(qv[d0 / 64], 2 * i) * ka;
        x += of_lane(qv[d0 / 64], 2 * i + 1) * kb;
      }
    }
    x *= a.scale * 1.44269504088896340736f;
    float next = fmaxf(top, lane < n ? x : top);
#pragma unroll
    for (int m = 1; m < WAVE; m *= 2) next = fmaxf(next, __shfl_xor(next, m));
    const float by = __builtin_amdgcn_exp2f(top - next);
    const float e = lane < n ? __builtin_amdgcn_exp2f(x - next - 30.0f) : 0.0f;  // as bf16's reference (ops.hpp)
    top = next;
    float total = e;
#pragma unroll
    for (int m = 1; m < WAVE; m *= 2) total += __shfl_xor(total, m);
    den = den * by + total;
#pragma unroll
    for (int d = 0; d < ND; ++d) acc[d] = weighted(acc[d], by);
    const uint16_t* v = vbase + k0 * a.v_strides.row + lane;
    auto values = [&](auto small) INLINE {  // small: some weights are too small for 32 bits
      for (int i0 = 0; i0 < n; i0 += AT_ONCE) {
        uint16_t w[AT_ONCE][ND];
#pragma unroll
        for (int i = 0; i < AT_ONCE; ++i)
#pragma unroll
          for (int d = 0; d < ND; ++d) w[i][d] = v[min(i0 + i, n - 1) * a.v_strides.row + d * WAVE];
#pragma unroll
        for (int i = 0; i < AT_ONCE; ++i) {
          const float f = of_lane(e, min(i0 + i, n - 1));
#pragma unroll
          for (int d = 0; d < ND; ++d) {
            float y;
            unpack2<TYPE>(w[i][d], y, unused);
            if constexpr (small) y = weighted(y, f);
            else y *= f;
            acc[d] += i0 + i < n ? y : 0.0f;
          }
        }
      }
    };
    if (__ballot(lane < n && e == 0)) values(std::true_type());
    else values(std::false_type());
  }
#pragma unroll
  for (int d = 0; d < ND; ++d)
    ((uint16_t*)a.out)[at * D + d * WAVE + lane] = (uint16_t)pack2<TYPE>(den == 0 ? 0.0f : acc[d] / den, 0.0f);
  if (a.lse && lane == 0) a.lse[at] = log_sum(top + 30.0f, den);
}

template <int TYPE, int D, int WAVES, bool VEC, bool SPLIT>
__global__ __launch_bounds__(WAVES * WAVE, 2) void k_prompt(PromptArgs p) {
  constexpr int QROWS = 32 * WAVES, THREADS = WAVE * WAVES;
  const herschel_prompt_args& a = p.a;
  constexpr int NC = D / 8;    // 16-byte chunks of a K row
  constexpr int DT = D / 32;   // blocks of dimensions
  constexpr int NS = D / 16;   // steps of the first product
  constexpr int KBYTES = KT * D * 2;
  constexpr int VBUFS = WAVES == 8 ? 3 : 2;
  __shared__ __align__(16) char s_k[3 * KBYTES];
  __shared__ __align__(16) char s_v[VBUFS * KBYTES];

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
  if (level == 0 && qh == 0 && tid == 0 &&
      (q0 != q0w || (b == 0 && q0 > 0) || q1 != q1w || kk0 != k0w || kk1 != k1w || q1 - q0 != nq))
    flag(a.status, HERSCHEL_OP_BAD_LENGTH);
  if (!SPLIT || blockIdx.y == 0) rows_without<D>(a, b, q0w, q1w, q0, q1, nq, qh, 1, level, p.levels);
  const int row0 = level * QROWS;
  if (row0 >= nq) return;
  const int kh = qh / p.group;
  const int shift = nk - (int)(q1 - q0);  // causal: row i sees keys up to i + shift

  // this lane's query row, and the keys it sees: [from, to)
  const int row = row0 + wave * 32 + n;
  const int to = row >= nq ? 0 : a.causal ? min(nk, max(0, row + shift + 1)) : nk;
  const int from = window_from(row + shift, a.window);
  // the workgroup's
  const int last = min(row0 + QROWS, nq) - 1;
  const int wg_to = a.causal ? min(nk, max(0, last + shift + 1)) : nk;
  int wg_from = min(wg_to, window_from(row0 + shift, a.window)) / KT * KT;
  int tiles = (wg_to - wg_from + KT - 1) / KT;
  if constexpr (SPLIT) {
    const int begin = (int)((int64_t)tiles * blockIdx.y / p.splits);
    tiles = (int)((int64_t)tiles * (blockIdx.y + 1) / p.splits) - begin;
    wg_from += begin * KT;
  }
  // keys outside these may be hidden from a row of this wave
  const int first_row = row0 + wave * 32;
  const int all_to = first_row + 32 > nq ? 0 : a.causal ? min(nk, max(0, first_row + shift + 1)) : nk;
  const int all_from = window_from(first_row + 31 + shift, a.window);
  // keys outside these are hidden from all rows of the wave
  const int any_to = a.causal ? min(nk, max(0, first_row + 32 + shift)) : nk;
  const int any_from = window_from(first_row + shift, a.window);

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

  // A thread's share of a tile: chunks of 16 bytes, by rows.  LDS chunk c of a
  // row holds the row's chunk c ^ f(row): f is the row's number for K; for V a
  // multiple of four that differs where rows that are read together would meet.
  constexpr int KL = KT * NC / THREADS;
  constexpr int ROWS = THREADS / NC;  // rows of one chunk a thread: f repeats after them
  const uint16_t* kbase = (const uint16_t*)a.k + kk0 * a.k_strides.row + kh * a.k_strides.head;
  const uint16_t* vbase = (const uint16_t*)a.v + kk0 * a.v_strides.row + kh * a.v_strides.head;
  auto fk = [](int r) INLINE { return (D == 128 ? r : r >> 1) & (NC - 1); };
  auto fv = [](int r) INLINE { return D == 128 ? (r & 3) * 4 : (r >> 1 & 1) * 4; };
  const int crow = tid / NC, cc = tid % NC;
  // whole tiles: one 32-bit offset a thread from addresses that are the workgroup's
  const uint32_t koff = (uint32_t)(crow * a.k_strides.row + (cc ^ fk(crow)) * 8) * 2;
  const uint32_t voff = (uint32_t)(crow * a.v_strides.row + (cc ^ fv(crow)) * 8) * 2;
  auto load_rows = [&](const uint16_t* base, int64_t stride, uint32_t off, int swap, char* dst, int tile) INLINE {
    const int k0 = wg_from + tile * KT;
    dst += wave * WAVE * 16;
    if (VEC && k0 + KT <= nk) {
      const char* src = (const char*)(base + (int64_t)k0 * stride);
#pragma unroll
      for (int i = 0; i < KL; ++i) copy_to_lds(src + (int64_t)(i * ROWS) * stride * 2 + off, dst + i * (THREADS * 16));
    } else {  // rows past the sequence's end read its last row
      for (int i = 0; i < KL; ++i) {
        const uint16_t* src = base + min(k0 + crow + i * ROWS, nk - 1) * stride + swap * 8;
        *(u32x4*)(dst + i * (THREADS * 16) + lane * 16) = VEC ? *(const u32x4*)src : load_elements(src);
      }
    }
  };
  auto load_k = [&](int tile, char* to) INLINE { load_rows(kbase, a.k_strides.row, koff, cc ^ fk(crow), to, tile); };
  auto load_v = [&](int tile, char* to) INLINE { load_rows(vbase, a.v_strides.row, voff, cc ^ fv(crow), to, tile); };
  // operands: step s of the keys of half h of a tile; dimension block d, step s of the keys of half h
  auto read_k = [&](const char* k, int h, int s) INLINE {
    return *(const u32x4*)(k + (32 * h + n) * (D * 2) + (((2 * s + g) ^ fk(n)) * 16));
  };
  // Lane l of 16 reads four dimensions of key l / 4 of four; it receives
  // dimension l of all four keys.
  const int vrow = 4 * g + lane % 16 / 4, vcol = 2 * (lane / 16 % 2) + lane % 4 / 2;
  auto read_v = [&](const char* v, int h, int d, int s) INLINE {
    u32x4 r;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int key = 32 * h + 16 * s + 8 * i + vrow;
      const char* at = v + key * (D * 2) + ((4 * d + vcol) ^ fv(vrow)) * 16 + lane % 2 * 8;
      const u32x2 w = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsHalves*)at));
      r[2 * i] = w[0];
      r[2 * i + 1] = w[1];
    }
    return r;
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

  auto hidden = [&](int t) INLINE { return wg_from + t * KT >= any_to || wg_from + (t + 1) * KT <= any_from; };
  auto masked = [&](int t) INLINE { return wg_from + (t + 1) * KT > all_to || wg_from + t * KT < all_from; };
  auto scores = [&](const char* kc) INLINE {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      f32x16 zero;
#pragma unroll
      for (int i = 0; i < 16; ++i) zero[i] = 0;
      sc[h] = mfma32<TYPE>(read_k(kc, h, 0), q[0], zero);
#pragma unroll
      for (int s = 1; s < NS; ++s) sc[h] = mfma32<TYPE>(read_k(kc, h, s), q[s], sc[h]);
    }
    reads_ahead<2 * NS, 1, 0>();
  };
  // a wave's first tile moves the reference in any case
  auto softmax = [&](int t, bool first) INLINE {
    if (masked(t)) {
      const int k0 = wg_from + t * KT, lo = from - k0 - 4 * g, hi = to - k0 - 4 * g;
#pragma unroll
      for (int i = 0; i < 32; ++i) {
        const int c = 32 * (i / 16) + 8 * (i % 16 / 4) + i % 4;
        sc[i / 16][i % 16] = c < hi ? sc[i / 16][i % 16] : -INFINITY;
      }
      if (a.window > 0)
#pragma unroll
        for (int i = 0; i < 32; ++i) {
          const int c = 32 * (i / 16) + 8 * (i % 16 / 4) + i % 4;
          sc[i / 16][i % 16] = c >= lo ? sc[i / 16][i % 16] : -INFINITY;
        }
    }
    float s = 0;
    if (!first) s = exponentials();
    if (first || Reference<TYPE>::template off<2>(s)) {
      float top = sc[0][0];
#pragma unroll
      for (int i = 1; i < 32; ++i) top = fmaxf(top, sc[i / 16][i % 16]);
      top = fmaxf(top, __shfl_xor(top, 32));
      const float next = Reference<TYPE>::moved(ref, top * to_log2, sum + __shfl_xor(sum, 32));
      const float by = __builtin_amdgcn_exp2f(ref - next);
      ref = next;
      sum *= by;
#pragma unroll
      for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[d][i] *= by;
      s = exponentials();
    }
    sum += s;
  };
  auto product = [&](const char* vc) INLINE {
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
      for (int k = 0; k < 4; ++k) o[d] = mfma32<TYPE>(read_v(vc, k / 2, d, k % 2), pb[k], o[d]);
    reads_ahead<4 * DT, 2, 1>();
  };
  // The workgroup's waves meet; this wave's copies but the newest `keep` are done.
  auto meet = [&](int keep) INLINE {
    asm volatile("" ::: "memory");
    if (keep == 0) __builtin_amdgcn_s_waitcnt(0x0070);  // vmcnt, lgkmcnt 0
    else if (keep == KL) __builtin_amdgcn_s_waitcnt(0x0070 | KL);
    else __builtin_amdgcn_s_waitcnt(0xc07f);            // lgkmcnt 0
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
  };
  // Copies asked for before this are asked for before those after it: `meet` counts by their order, which nothing else
  // in the source holds (they go to different buffers).
  auto in_order = []() INLINE { asm volatile("" ::: "memory"); };
  if (tiles > 0) {
    if constexpr (WAVES == 4) {
      load_k(0, s_k);
      load_v(0, s_v);
      in_order();
      if (tiles > 1) load_k(1, s_k + KBYTES);
      meet(tiles > 1 ? KL : 0);
      bool first = true;
      // Tile t, from kc and vc, while later tiles are copied to kn and vn: the
      // pointers' restrict is what lets reads pass copies still under way.
      auto work = [&](int t, const char* __restrict kc, const char* __restrict vc, char* __restrict kn,
                      char* __restrict vn) INLINE {
        if (t + 1 < tiles) load_v(t + 1, vn);
        in_order();  // the newest KL copies are K's: those that may be under way when the waves meet
        if (t + 2 < tiles) load_k(t + 2, kn);
        if (!hidden(t)) {
          scores(kc);
          softmax(t, first);
          product(vc);
          first = false;
        }
      };
      int kb0 = 0, kb1 = 1, kb2 = 2;  // K's buffers of tiles t, t + 1, t + 2
      for (int t = 0; t < tiles; ++t) {
        work(t, s_k + kb0 * KBYTES, s_v + (t & 1) * KBYTES, s_k + kb2 * KBYTES, s_v + (~t & 1) * KBYTES);
        meet(t + 2 < tiles ? KL : 0);
        const int x = kb0;
        kb0 = kb1;
        kb1 = kb2;
        kb2 = x;
      }
    } else {
      load_k(0, s_k);
      load_v(0, s_v);
      if (tiles > 1) load_k(1, s_k + KBYTES), load_v(1, s_v + KBYTES);
      if (tiles > 2) load_k(2, s_k + 2 * KBYTES);
      meet(0);
      if (!hidden(0)) {
        scores(s_k);
        softmax(0, true);
      }
      // The first four waves (one a SIMD) and the last four take turns: while one
      // half runs the products of a step, the other runs the exponentials.
      const bool second = wave >= 4;
      if (second) meet(-1);
      int b0 = 0, b1 = 1, b2 = 2;  // buffers of tiles t, t + 1, t + 2
      for (int t = 0; t < tiles; ++t) {
        __builtin_amdgcn_s_setprio(1);
        if (t + 1 < tiles && !hidden(t + 1)) scores(s_k + b1 * KBYTES);
        if (!hidden(t)) product(s_v + b0 * KBYTES);
        __builtin_amdgcn_s_setprio(0);
        meet(-1);
        if (t + 3 < tiles) load_k(t + 3, s_k + b0 * KBYTES);
        if (t + 2 < tiles) load_v(t + 2, s_v + b2 * KBYTES);
        if (t + 1 < tiles && !hidden(t + 1)) softmax(t + 1, false);
        meet(0);
        const int x = b0;
        b0 = b1;
        b1 = b2;
        b2 = x;
      }
      if (!second) meet(-1);
    }
  }

  sum += __shfl_xor(sum, 32);
  if constexpr (SPLIT) {
    if (row >= nq) return;
    float* part = row_part<D>(a, blockIdx.y, (q0 + row) * a.q_heads + qh);
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        *(f32x4*)(part + 32 * d + 8 * i + 4 * g) = f32x4{o[d][4 * i], o[d][4 * i + 1], o[d][4 * i + 2], o[d][4 * i + 3]};
    if (g == 0) part[D] = ref, part[D + 1] = sum;
    return;
  }
  float check = sum - sum;  // 0, or NaN if a sum is not finite
#pragma unroll
  for (int d = 0; d < DT; ++d)
#pragma unroll
    for (int i = 0; i < 16; ++i) check += o[d][i] - o[d][i];
  if (__ballot(!(check == 0))) {
    const int rows = min(32, nq - first_row);
    for (int r = 0; r < rows; ++r) {
      const int64_t at = (q0 + first_row + r) * a.q_heads + qh;
      row_by_key<TYPE, D>((const uint16_t*)a.q + (q0 + first_row + r) * a.q_strides.row + qh * a.q_strides.head, kbase, vbase,
                          a, __shfl(from, r), __shfl(to, r), at);
    }
    return;
  }
  if (row >= nq) return;
  const float inv = sum > 0 ? 1.0f / sum : 0.0f;  // no key seen: 0
  const int64_t at = (q0 + row) * a.q_heads + qh;
#pragma unroll
  for (int d = 0; d < DT; ++d)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      uint16_t* out = (uint16_t*)a.out + at * D + 32 * d + 8 * i + 4 * g;
      *(u32x2*)out = u32x2{pack2<TYPE>(o[d][4 * i] * inv, o[d][4 * i + 1] * inv),
                           pack2<TYPE>(o[d][4 * i + 2] * inv, o[d][4 * i + 3] * inv)};
    }
  if (a.lse && g == 0) a.lse[at] = log_sum(ref, sum);
}

// Few rows: 32 to a workgroup, whose four waves share the keys, 32 at a time.
//
// Where workgroups of 128 rows would leave most of the card idle, what counts is
// the chain of tiles that one wave goes through: here it is four times shorter
// (with 32 heads of 128, 128 rows 6.8 us against 9.0, 512 rows 13.1 against 17.1,
// 16 rows over 2048 keys 24 against 49).  The rows are a token's query heads
// of one key head, then the next token's, so that a call with fewer than 32
// tokens fills its workgroups too.  A key goes to one wave only, through LDS that
// is the wave's own (loads in the products' layout touch a row per lane: 2048
// keys took 25.8 us where this took 22.6), so no wave waits for another before the parts are joined.
// The next step's keys are asked for once the scores are there, its values after
// the second product.
//
// Packed sequences of different lengths would leave most workgroups of a grid of
// levels by sequences without rows, and one waits for the lengths to find that
// out: here the grid has the levels that the rows allow and one a sequence (8
// sequences of 1 to 600 tokens, 16 heads of 64: 25.4 to 10.5 us).  Workgroups of
// 128 rows have fewer levels, and the search cost them as much when tried (24 x 1
// to 300 tokens 10.5 against 11.8 us).
constexpr int FEW_WAVES = 4;  // eight: 16 rows over 2048 keys 17.9 us against 17.5, 512 rows 18.3 against 13.1
template <int TYPE, int D, bool VEC, bool SPLIT>
__global__ __launch_bounds__(FEW_WAVES * WAVE, 2) void k_prompt_few(PromptArgs p) {
  const herschel_prompt_args& a = p.a;
  constexpr int W = FEW_WAVES;
  constexpr int DT = D / 32, NS = D / 16;
  constexpr int NC = D / 8;          // 16-byte chunks of a row
  constexpr int PART = 16 * DT / W;  // values of a lane that a wave joins
  constexpr int BYTES = 32 * D * 2;
  // a wave's keys and values; at the end, the first and second half of its sums
  __shared__ __align__(16) char s_k[W * BYTES];
  __shared__ __align__(16) char s_v[W * BYTES];
  __shared__ float s_ref[W][32], s_sum[W][32];
  const int tid = threadIdx.x, lane = tid % WAVE, wave = __builtin_amdgcn_readfirstlane(tid / WAVE), n = lane % 32, g = lane / 32;
  uint32_t id = blockIdx.x;  // longest first
  const int kh = (int)(id % a.kv_heads);
  id /= a.kv_heads;
  int b = (int)(id % a.n_seqs), level = p.levels - 1 - (int)(id / a.n_seqs);
  int64_t q0, q1;
  if (p.packed) {
    if (blockIdx.x == 0 && tid < WAVE) report_lengths(a);
    if (a.cu_q[0] > 0 || a.cu_q[a.n_seqs] < a.n_q) {  // before the first sequence, after the last
      const int64_t first = min((int64_t)max(a.cu_q[0], 0), a.n_q);
      int64_t lo, hi;
      start_range(a, lo, hi);
      no_query<D>(a, 0, first, kh * p.group, p.group, id, gridDim.x / a.kv_heads);
      no_query<D>(a, max(first, hi), a.n_q, kh * p.group, p.group, id, gridDim.x / a.kv_heads);
    }
    if (!find_level(a, p.group, id, b, level, q0, q1)) return;
  }
  // lengths taken as the nearest valid
  const int64_t q0w = a.cu_q[b], q1w = a.cu_q[b + 1], k0w = a.cu_k[b], k1w = a.cu_k[b + 1];
  if (!p.packed) q0 = min(max(q0w, (int64_t)0), a.n_q), q1 = min(max(q1w, q0), a.n_q);
  const int64_t kk0 = min(max(k0w, (int64_t)0), a.n_k), kk1 = min(max(k1w, kk0), a.n_k);
  const int nq = (int)min(q1 - q0, (int64_t)a.max_q), nk = (int)(kk1 - kk0);
  const int row0 = level * 32, rows = nq * p.group;
  if (p.packed) {
    if (q1 - q0 > nq) no_query<D>(a, q0 + nq, q1, kh * p.group, p.group, level, (rows + 31) / 32);
  } else {
    if (level == 0 && kh == 0 && tid == 0 &&
        (q0 != q0w || (b == 0 && q0 > 0) || q1 != q1w || kk0 != k0w || kk1 != k1w || q1 - q0 != nq))
      flag(a.status, HERSCHEL_OP_BAD_LENGTH);
    if (!SPLIT || blockIdx.y == 0) rows_without<D>(a, b, q0w, q1w, q0, q1, nq, kh * p.group, p.group, level, p.levels);
  }
  if (row0 >= rows) return;
  const int shift = nk - (int)(q1 - q0);  // causal: token i sees keys up to i + shift

  // this lane's row (the last one again past it), and the keys it sees: [from, to)
  const int row = min(row0 + n, rows - 1), tok = row / p.group, qh = kh * p.group + row % p.group;
  auto sees_to = [&](int t) INLINE { return a.causal ? min(nk, max(0, t + shift + 1)) : nk; };
  auto sees_from = [&](int t) INLINE { return window_from(t + shift, a.window); };
  const int to = sees_to(tok), from = sees_from(tok);
  // the workgroup's
  const int first = row0 / p.group, last = min(row0 + 31, rows - 1) / p.group;
  const int any_to = sees_to(last), any_from = sees_from(first), all_to = sees_to(first), all_from = sees_from(last);

  const uint16_t* qrow = (const uint16_t*)a.q + (q0 + tok) * a.q_strides.row + qh * a.q_strides.head;
  const uint32_t sign = a.scale < 0 ? 0x80008000u : 0u;
  u32x4 q[NS];
#pragma unroll
  for (int s = 0; s < NS; ++s) q[s] = VEC ? *(const u32x4*)(qrow + 16 * s + 8 * g) : load_elements(qrow + 16 * s + 8 * g);
  const float to_log2 = fmaxf(fabsf(a.scale) * 1.44269504088896340736f, 0x1p-100f);
  const uint16_t* kbase = (const uint16_t*)a.k + kk0 * a.k_strides.row + kh * a.k_strides.head;
  const uint16_t* vbase = (const uint16_t*)a.v + kk0 * a.v_strides.row + kh * a.v_strides.head;

  f32x16 o[DT];
#pragma unroll
  for (int d = 0; d < DT; ++d)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[d][i] = 0;
  float ref = NO_KEY, sum = 0;
  // A load takes RPC whole rows; LDS chunk c of a row holds the row's chunk
  // c ^ f(row), as above.
  constexpr int RPC = WAVE / NC, LOADS = 32 / RPC;
  auto fk = [](int r) INLINE { return (D == 128 ? r : r >> 1) & (NC - 1); };
  auto fv = [](int r) INLINE { return D == 128 ? (r & 3) * 4 : (r >> 1 & 1) * 4; };
  char* const my_k = s_k + wave * BYTES;
  char* const my_v = s_v + wave * BYTES;
  const int crow = lane / NC, cc = lane % NC;
  const uint32_t koff = (uint32_t)(crow * a.k_strides.row + cc * 8) * 2;
  const uint32_t voff = (uint32_t)(crow * a.v_strides.row + cc * 8) * 2;
  auto load = [&](u32x4 (&to)[LOADS], const uint16_t* base, int64_t stride, uint32_t off, int k0) INLINE {
    if (VEC && k0 + 32 <= nk) {
      const char* src = (const char*)(base + k0 * stride);
#pragma unroll
      for (int i = 0; i < LOADS; ++i) to[i] = *(const u32x4*)(src + i * RPC * stride * 2 + off);
    } else {  // rows past the sequence's end read its last row
#pragma unroll
      for (int i = 0; i < LOADS; ++i) {
        const uint16_t* src = base + min(k0 + i * RPC + crow, nk - 1) * stride + cc * 8;
        to[i] = VEC ? *(const u32x4*)src : load_elements(src);
      }
    }
  };
  // LDS written by the wave is read by its other lanes
  auto written = [&]() INLINE {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront", "local");
    __builtin_amdgcn_wave_barrier();
  };
  u32x4 k[LOADS], v[LOADS];
  const int vrow = 4 * g + lane % 16 / 4, vcol = 2 * (lane / 16 % 2) + lane % 4 / 2;
  int begin = any_from / 32 * 32, end = any_to;
  if constexpr (SPLIT) {
    const int steps = max(0, end - begin + 31) / 32;
    end = min(end, begin + 32 * (int)((int64_t)steps * (blockIdx.y + 1) / p.splits));
    begin += 32 * (int)((int64_t)steps * blockIdx.y / p.splits);
  }
  int k0 = begin + wave * 32;
  if (k0 < end) {
    load(k, kbase, a.k_strides.row, koff, k0);
    load(v, vbase, a.v_strides.row, voff, k0);
  }
#pragma unroll
  for (int s = 0; s < NS; ++s) q[s] ^= sign;  // a negative scale goes into Q's signs: what is left is not negative
  for (; k0 < end; k0 += 32 * W) {
    f32x16 sc;
#pragma unroll
    for (int i = 0; i < 16; ++i) sc[i] = 0;
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
      const int r = i * RPC + crow;
      *(u32x4*)(my_k + r * (D * 2) + (cc ^ fk(r)) * 16) = k[i];
    }
    written();
#pragma unroll
    for (int s = 0; s < NS; ++s)
      sc = mfma32<TYPE>(*(const u32x4*)(my_k + n * (D * 2) + (((2 * s + g) ^ fk(n)) * 16)), q[s], sc);
    const bool more = k0 + 32 * W < end;
    if (more) load(k, kbase, a.k_strides.row, koff, k0 + 32 * W);
    if (k0 + 32 > all_to || k0 < all_from) {
      const int lo = from - k0 - 4 * g, hi = to - k0 - 4 * g;
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int c = 8 * (i / 4) + i % 4;
        sc[i] = c < hi ? sc[i] : -INFINITY;
      }
      if (a.window > 0)
#pragma unroll
        for (int i = 0; i < 16; ++i) sc[i] = 8 * (i / 4) + i % 4 >= lo ? sc[i] : -INFINITY;
    }
    u32x4 pb[2];
    auto exponentials = [&]() INLINE {
      float s = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float e0 = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[2 * i], to_log2, -ref));
        const float e1 = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[2 * i + 1], to_log2, -ref));
        s += e0 + e1;
        pb[i / 4][i % 4] = pack2<TYPE>(e0, e1);
      }
      return s;
    };
    const bool first = k0 == begin + wave * 32;  // moves the reference in any case
    float t = 0;
    if (!first) t = exponentials();
    if (first || Reference<TYPE>::template off<2>(t)) {
      float top = sc[0];
#pragma unroll
      for (int i = 1; i < 16; ++i) top = fmaxf(top, sc[i]);
      top = fmaxf(top, __shfl_xor(top, 32));
      const float next = Reference<TYPE>::moved(ref, top * to_log2, sum + __shfl_xor(sum, 32));
      const float by = __builtin_amdgcn_exp2f(ref - next);
      ref = next;
      sum *= by;
#pragma unroll
      for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[d][i] *= by;
      t = exponentials();
    }
    sum += t;
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
      const int r = i * RPC + crow;
      *(u32x4*)(my_v + r * (D * 2) + (cc ^ fv(r)) * 16) = v[i];
    }
    written();
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        u32x4 vt;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const int key = 16 * s + 8 * i + vrow;
          const char* at = my_v + key * (D * 2) + ((4 * d + vcol) ^ fv(vrow)) * 16 + lane % 2 * 8;
          const u32x2 w = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsHalves*)at));
          vt[2 * i] = w[0];
          vt[2 * i + 1] = w[1];
        }
        o[d] = mfma32<TYPE>(vt, pb[s], o[d]);
      }
    written();
    if (more) load(v, vbase, a.v_strides.row, voff, k0 + 32 * W);
  }
  // The waves' parts, joined through LDS: wave w the values w PART ... of every lane.
  sum += __shfl_xor(sum, 32);
#pragma unroll
  for (int d = 0; d < DT; ++d)
#pragma unroll
    for (int i = 0; i < 16; ++i) ((float*)(d < DT / 2 ? my_k : my_v))[(d % (DT / 2) * 16 + i) * WAVE + lane] = o[d][i];
  if (g == 0) {
    s_ref[wave][n] = ref;
    s_sum[wave][n] = sum;
  }
  __syncthreads();
  float acc[PART], den = 0, top = NO_KEY;
#pragma unroll
  for (int w = 0; w < W; ++w) top = fmaxf(top, s_ref[w][n]);
#pragma unroll
  for (int i = 0; i < PART; ++i) acc[i] = 0;
#pragma unroll
  for (int w = 0; w < W; ++w) {
    const float by = __builtin_amdgcn_exp2f(s_ref[w][n] - top);
    den += s_sum[w][n] * by;
#pragma unroll
    for (int i = 0; i < PART; ++i)
      acc[i] += ((const float*)((wave < W / 2 ? s_k : s_v) + w * BYTES))[(wave % (W / 2) * PART + i) * WAVE + lane] * by;
  }
  const int64_t at = (q0 + tok) * a.q_heads + qh;
  if constexpr (SPLIT) {
    if (row0 + n >= rows) return;
    float* part = row_part<D>(a, blockIdx.y, at);
#pragma unroll
    for (int i = 0; i < PART; i += 4) {
      const int x = wave * PART + i;
      *(f32x4*)(part + 32 * (x / 16) + 8 * (x % 16 / 4) + 4 * g) = f32x4{acc[i], acc[i + 1], acc[i + 2], acc[i + 3]};
    }
    if (g == 0 && wave == 0) part[D] = top, part[D + 1] = den;
    return;
  }
  float check = den - den;  // 0, or NaN if a sum is not finite
#pragma unroll
  for (int i = 0; i < PART; ++i) check += acc[i] - acc[i];
  if (__syncthreads_or(!(check == 0))) {
    for (int r = row0 + wave; r < min(row0 + 32, rows); r += W) {
      const int t = r / p.group, h = kh * p.group + r % p.group;
      row_by_key<TYPE, D>((const uint16_t*)a.q + (q0 + t) * a.q_strides.row + h * a.q_strides.head, kbase, vbase, a,
                          sees_from(t), sees_to(t), (q0 + t) * a.q_heads + h);
    }
    return;
  }
  if (row0 + n >= rows) return;
  const float inv = den > 0 ? 1.0f / den : 0.0f;  // no key seen: 0
#pragma unroll
  for (int i = 0; i < PART; i += 4) {  // four dimensions in order
    const int x = wave * PART + i;
    uint16_t* out = (uint16_t*)a.out + at * D + 32 * (x / 16) + 8 * (x % 16 / 4) + 4 * g;
    *(u32x2*)out = u32x2{pack2<TYPE>(acc[i] * inv, acc[i + 1] * inv), pack2<TYPE>(acc[i + 2] * inv, acc[i + 3] * inv)};
  }
  if (a.lse && g == 0 && wave == 0) a.lse[at] = log_sum(top, den);
}

// Joins the parts of each row: a wave per row, four rows in turn.
constexpr int JOIN_ROWS = 16;
constexpr int MAX_SPLITS = 16;
template <int TYPE, int D>
__global__ __launch_bounds__(256) void k_prompt_join(PromptArgs p) {
  const herschel_prompt_args& a = p.a;
  constexpr int ND = D / WAVE;
  const int lane = threadIdx.x % WAVE, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / WAVE);
  const int b = (int)(blockIdx.x % a.n_seqs);
  const int64_t x0 = (int64_t)(blockIdx.x / a.n_seqs) * JOIN_ROWS;
  // lengths taken as the nearest valid
  const int64_t q0 = min(max((int64_t)a.cu_q[b], (int64_t)0), a.n_q), q1 = min(max((int64_t)a.cu_q[b + 1], q0), a.n_q);
  const int64_t kk0 = min(max((int64_t)a.cu_k[b], (int64_t)0), a.n_k), kk1 = min(max((int64_t)a.cu_k[b + 1], kk0), a.n_k);
  const int64_t rows = min(q1 - q0, (int64_t)a.max_q) * a.q_heads;
  const int nk = (int)(kk1 - kk0), shift = nk - (int)(q1 - q0);
  for (int64_t x = x0 + wave; x < min(x0 + JOIN_ROWS, rows); x += 4) {
    const int64_t at = q0 * a.q_heads + x;
    float r = NO_KEY, t = 0;
    if (lane < p.splits) {
      const float* part = row_part<D>(a, lane, at);
      r = part[D], t = part[D + 1];
    }
    float v[MAX_SPLITS][ND];
#pragma unroll
    for (int i = 0; i < MAX_SPLITS; ++i)
      if (i < p.splits)
#pragma unroll
        for (int d = 0; d < ND; ++d) v[i][d] = row_part<D>(a, i, at)[lane * ND + d];
    float top = r;
#pragma unroll
    for (int m = 1; m < MAX_SPLITS; m *= 2) top = fmaxf(top, __shfl_xor(top, m));
    top = __builtin_bit_cast(float, __builtin_amdgcn_readfirstlane(__builtin_bit_cast(int, top)));
    const float by = __builtin_amdgcn_exp2f(r - top);
    float den = 0, acc[ND];
#pragma unroll
    for (int d = 0; d < ND; ++d) acc[d] = 0;
#pragma unroll
    for (int i = 0; i < MAX_SPLITS; ++i)
      if (i < p.splits) {
        const float f = __shfl(by, i);
        den += __shfl(t, i) * f;
#pragma unroll
        for (int d = 0; d < ND; ++d) acc[d] += v[i][d] * f;
      }
    float check = den - den;  // 0, or NaN if a sum is not finite
#pragma unroll
    for (int d = 0; d < ND; ++d) check += acc[d] - acc[d];
    if (__ballot(!(check == 0))) {
      const int tok = (int)(x / a.q_heads), qh = (int)(x % a.q_heads), kh = qh / p.group;
      row_by_key<TYPE, D>((const uint16_t*)a.q + (q0 + tok) * a.q_strides.row + qh * a.q_strides.head,
                          (const uint16_t*)a.k + kk0 * a.k_strides.row + kh * a.k_strides.head,
                          (const uint16_t*)a.v + kk0 * a.v_strides.row + kh * a.v_strides.head, a,
                          window_from(tok + shift, a.window),
                          a.causal ? min(nk, max(0, tok + shift + 1)) : nk, at);
      continue;
    }
    const float inv = den > 0 ? 1.0f / den : 0.0f;  // no key seen: 0
    uint16_t* out = (uint16_t*)a.out + at * D + lane * ND;
    if constexpr (ND == 2) *(uint32_t*)out = pack2<TYPE>(acc[0] * inv, acc[1] * inv);
    else *out = (uint16_t)pack2<TYPE>(acc[0] * inv, 0.0f);
    if (a.lse && lane == 0) a.lse[at] = log_sum(top, den);
  }
}

template <int TYPE, int D>
static int prompt_join(PromptArgs& p) {
  const int64_t blocks = ((int64_t)p.a.max_q * p.a.q_heads + JOIN_ROWS - 1) / JOIN_ROWS * p.a.n_seqs;
  if (blocks > 0x7fffffff) return HERSCHEL_EINVAL;
  return launch(k_prompt_join<TYPE, D>, dim3((unsigned)blocks), dim3(256), 0, p.a.hip_stream, p);
}

// Packed: where a quarter of the grid is left, and the sequences are found in two rounds of
// the scan (4 heads of 64: 32 x 1 to 300 tokens 12.5 to 7.6 us, 64 x 1 to 300 14.0
// to 8.8; 3 x 100 to 900 of 16 heads, half the grid, would take 12.4 against 11.6, 200 x
// 1 to 60 8.3 against 8.0, 400 x 1 to 20 9.9 against 7.2).
constexpr int PACKED_SEQS = 128;

template <int TYPE, int D>
static int prompt_few(PromptArgs& p, bool vec) {
  const int64_t levels = std::max<int64_t>(1, ((int64_t)p.a.max_q * p.group + 31) / 32), most = p.a.n_q * p.group / 32 + p.a.n_seqs;
  p.packed = p.a.max_q > 0 && p.a.n_seqs > 1 && p.a.n_seqs <= PACKED_SEQS && p.splits == 1 && 4 * most <= levels * p.a.n_seqs;
  const int64_t blocks = (p.packed ? most : levels * p.a.n_seqs) * p.a.kv_heads;
  if (blocks > 0x7fffffff) return HERSCHEL_EINVAL;
  p.levels = (int)levels;
  auto kernel = vec ? p.splits > 1 ? k_prompt_few<TYPE, D, true, true> : k_prompt_few<TYPE, D, true, false>
                    : p.splits > 1 ? k_prompt_few<TYPE, D, false, true> : k_prompt_few<TYPE, D, false, false>;
  const int rc = launch(kernel, dim3((unsigned)blocks, p.splits), dim3(FEW_WAVES * WAVE), 0, p.a.hip_stream, p);
  return rc == HERSCHEL_OK && p.splits > 1 ? prompt_join<TYPE, D>(p) : rc;
}

template <int TYPE, int D, int WAVES>
static int prompt_launch(PromptArgs& p, bool vec) {
  p.levels = std::max(1, (p.a.max_q + 32 * WAVES - 1) / (32 * WAVES));
  // XCDs that share a key head: only where key heads and XCDs divide evenly
  const int G = p.a.kv_heads;
  p.spread = G >= 8 ? (G % 8 == 0 ? 1 : 0) : (8 % G == 0 ? 8 / G : 0);
  int64_t blocks = (int64_t)p.levels * p.a.n_seqs * p.a.q_heads;
  if (p.spread) blocks = (blocks / (G < 8 ? G : 8) + p.spread - 1) / p.spread * 8;
  if (blocks > 0x7fffffff) return HERSCHEL_EINVAL;
  if constexpr (WAVES == 4)
    if (p.splits > 1) {
      const int rc = launch(vec ? k_prompt<TYPE, D, 4, true, true> : k_prompt<TYPE, D, 4, false, true>,
                            dim3((unsigned)blocks, p.splits), dim3(4 * WAVE), 0, p.a.hip_stream, p);
      return rc == HERSCHEL_OK ? prompt_join<TYPE, D>(p) : rc;
    }
  return launch(vec ? k_prompt<TYPE, D, WAVES, true, false> : k_prompt<TYPE, D, WAVES, false, false>, dim3((unsigned)blocks),
                dim3(WAVES * WAVE), 0, p.a.hip_stream, p);
}

// What a call runs as, from its sizes and types alone (lengths are on the device:
// sequences count as their mean).  Times are of calls in a graph, causal, key heads
// a quarter of the heads; heads of 64 in half.
//
// Few rows: as long as 32 of them (of one key head) a workgroup make no more
// workgroups than the card holds at once, about 20,000 rows in all (24 x 16 rows
// of 16 heads of 64 5.2 us against 6.0, 512 rows of 32 heads of 128 13.1 against
// 17.1; 1024 rows of 32 heads of 128 28.8 against 26.5).  Over many keys workgroups
// of 128 rows read them fewer times, so rows times keys times dimensions have a
// limit too (of 128, 4 x 64 rows of 32 heads over 4096 keys, 4.3e9, 46 against 50,
// 512 rows, 8.6e9, 59 against 59; 777 rows of 8 heads over 12000 89 against 64; of
// 64, 4096 rows of 4 heads, 4.3e9, 30 against 42).  Heads of 64 gain up to 960
// workgroups (16 heads: 24 x 1 to 300 tokens 9.3 us against 11.2, 100 to 900 three
// times 11.6 against 21.9, 900 twice 16.5 against 22.1, one of 1800 21.7 against
// 38.8, though 24 x 64 7.0 against 6.4; 24 x 100, 1296 workgroups, 11.5 against 8.7).
//
// Else eight waves (256 rows) or four (128).  Eight in turns are faster where there
// is enough for every CU twice over: 4096 rows of 32 heads of 128 139 us against
// 151, 8192 twice 985 against 1063; below, what counts is more and smaller
// workgroups: 512 rows 21.5 against 17.1 us, 8 heads of 4096 95 against 81.  With
// heads of 64 the exponentials take longer than the products and turns lost when
// tried (4096 rows twice: 186 against 175 us).
//
// Parts: where the workgroups would not fill the card and keys are many, each
// workgroup's keys go to several.  The second launch and the parts' way through
// memory take 5 to 10 us.  Of few rows, four parts or more unless keys are very
// many: 16 rows of 32 heads over 2048 keys 17.5 us against 23.9, over 8192 24
// against 80; in two parts 2048 rows of 4 heads would take 30 against 24.  Of many,
// from 4096 keys on, to fill the card's places for workgroups once, or twice in up
// to four parts: 8192 rows of 4 heads 121 against 157, 4096 of 8 81 against 82, 512
// of 32 over 8192 keys 92 against 159 (in eight parts 103); 2048 rows of 16 heads
// would take 62 against 45.
struct PromptPlan {
  int waves;  // 0: few rows
  int splits;
  size_t bytes;
};
static PromptPlan prompt_plan(int64_t n_seqs, int64_t n_q, int64_t n_k, int64_t max_q, int64_t q_heads, int64_t kv_heads, int D) {
  PromptPlan plan{4, 1, 0};
  const int64_t rows = std::max<int64_t>(1, n_q / n_seqs), keys = n_k / n_seqs;
  int64_t splits = 1;
  const int64_t few = (n_q * (q_heads / kv_heads) / 32 + n_seqs) * kv_heads;  // workgroups of 32 rows, at most
  if ((n_q * q_heads <= 20480 || (D == 64 && few <= 960 && n_seqs <= PACKED_SEQS)) && n_q * q_heads * keys <= (5ll << 30) / D && max_q * (q_heads / kv_heads) < 0x7fffffe0) {
    plan.waves = 0;
    splits = std::min<int64_t>(512 / std::max<int64_t>(1, (n_q * q_heads + 31) / 32), keys / 512);
    if (splits < 4 && keys < 8192) splits = 1;
  } else if (D == 128 && rows >= 1024 && rows / 256 * n_seqs * q_heads >= 512) {
    plan.waves = 8;
  } else if (keys >= 4096) {
    const int64_t groups = (rows + 127) / 128 * n_seqs * q_heads;
    splits = std::min(std::max(512 / groups, std::min<int64_t>(1024 / groups, 4)), keys / 1024);
  }
  if (splits > 1) {
    plan.splits = (int)std::min<int64_t>(splits, MAX_SPLITS);
    plan.bytes = (size_t)plan.splits * n_q * q_heads * (D + 4) * 4;
  }
  return plan;
}

template <int TYPE, int D>
static int prompt_size(PromptArgs& p, const PromptPlan& plan, bool vec) {
  if (plan.waves == 0) return prompt_few<TYPE, D>(p, vec);
  if constexpr (D == 128)
    if (plan.waves == 8) return prompt_launch<TYPE, 128, 8>(p, vec);
  return prompt_launch<TYPE, D, 4>(p, vec);
}
template <int TYPE>
static int prompt_dim(PromptArgs& p, const PromptPlan& plan, bool vec) {
  return p.a.head_dim == 64 ? prompt_size<TYPE, 64>(p, plan, vec) : prompt_size<TYPE, 128>(p, plan, vec);
}

static bool prompt_sizes_ok(int32_t n_seqs, int64_t n_q, int64_t n_k, int32_t max_q, int32_t q_heads, int32_t kv_heads, int32_t head_dim) {
  return n_seqs >= 1 && n_q >= 0 && n_k >= 0 && max_q >= 0 && n_q <= 0x7fffffff && n_k <= 0x7fffffff &&
         (head_dim == 64 || head_dim == 128) && kv_heads >= 1 && q_heads >= 1 && q_heads % kv_heads == 0;
}

}  // namespace hop

extern "C" int herschel_attn_prompt_workspace(int32_t n_seqs, int64_t n_q, int64_t n_k, int32_t max_q, int32_t q_heads,
                                              int32_t kv_heads, int32_t head_dim, size_t* bytes) {
  using namespace hop;
  if (!bytes || !prompt_sizes_ok(n_seqs, n_q, n_k, max_q, q_heads, kv_heads, head_dim)) return HERSCHEL_EINVAL;
  *bytes = prompt_plan(n_seqs, n_q, n_k, std::min<int64_t>(max_q, n_q), q_heads, kv_heads, head_dim).bytes;
  return HERSCHEL_OK;
}

extern "C" int herschel_attn_prompt(const herschel_prompt_args* args) {
  using namespace hop;
  if (!args) return HERSCHEL_EINVAL;
  herschel_prompt_args a = *args;
  if (!prompt_sizes_ok(a.n_seqs, a.n_q, a.n_k, a.max_q, a.q_heads, a.kv_heads, a.head_dim) || !type_ok(a.type))
    return HERSCHEL_EINVAL;
  if (a.workspace && !aligned(a.workspace, 16)) return HERSCHEL_EWORKSPACE;
  if (a.window < 0 || !isfinite(a.scale) || !a.cu_q || !a.cu_k) return HERSCHEL_EINVAL;
  if (!strides_ok(a.q_strides) || !strides_ok(a.k_strides) || !strides_ok(a.v_strides)) return HERSCHEL_EINVAL;
  if ((a.n_q && (!a.q || !a.out || !aligned(a.q, 2) || !aligned(a.out, 8))) ||
      (a.n_k && (!a.k || !a.v || !aligned(a.k, 2) || !aligned(a.v, 2))))
    return HERSCHEL_EINVAL;
  if (a.n_q == 0) return HERSCHEL_OK;
  a.max_q = (int32_t)std::min<int64_t>(a.max_q, a.n_q);  // no sequence has more: grids and their arithmetic go by it
  PromptPlan plan = prompt_plan(a.n_seqs, a.n_q, a.n_k, a.max_q, a.q_heads, a.kv_heads, a.head_dim);
  if (!a.workspace || a.workspace_bytes < plan.bytes || a.max_q == 0) plan.splits = 1;
  PromptArgs p{a, a.q_heads / a.kv_heads, 0, 0, plan.splits, 0};
  // 16-byte loads, and a tile's rows within 31 bits of bytes
  const bool vec = a.k_strides.row < (1 << 23) && a.v_strides.row < (1 << 23) && chunks_aligned(a.q, a.q_strides) && chunks_aligned(a.k, a.k_strides) && chunks_aligned(a.v, a.v_strides);
  return a.type == HERSCHEL_BF16 ? prompt_dim<HERSCHEL_BF16>(p, plan, vec) : prompt_dim<HERSCHEL_F16>(p, plan, vec);
}
