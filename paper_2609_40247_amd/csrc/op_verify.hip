// Drafted tokens against the target's probabilities: how many are accepted, and
// the token drawn behind them.
//
// Only one row of the vocabulary a sequence is ever read, that of the first draft
// that is not accepted (and its counterpart of the draft's probabilities), found
// from the drafts' own probabilities, a few loads.  Up to ONE_ROW tokens a
// workgroup a sequence does it all: it sums what each wave's run of the row
// weighs, finds the run in which the cumulative sum passes the random number's,
// and in it the lane and the token.  Longer rows are summed in shares by many
// workgroups first; the second launch finds the share.  One launch is as fast as two
// at 32000 tokens of one sequence (8.3 us against 3.8 and 4.3) and takes 3 us less of the
// host; at 64000 it takes 14.8 against 3.8 and 4.4: its sums are 64-bit work of one CU.
// Large calls are bound by the sums' traffic: 64 sequences of 151936 tokens, 78 MB,
// 12.3 us, 6.3 TB/s, and 5.7 for the draw.
#include "ops.hpp"

namespace hop {

struct VerifyArgs {
  herschel_verify_args a;
  int shares;   // of a row
  int size;     // elements of a share, a multiple of SHARE_STEP
};

constexpr int VERIFY_THREADS = 256, VERIFY_WAVES = VERIFY_THREADS / WAVE;
constexpr int SHARE_STEP = VERIFY_THREADS * 8;
constexpr int MOST_STEPS = 16;  // of a share
constexpr int ONE_THREADS = 1024, ONE_ROW = ONE_THREADS * 8 * 4;

template <int TYPE>
__device__ __forceinline__ float probability(const void* p, int64_t at) {
  if constexpr (TYPE == HERSCHEL_F32) return ((const float*)p)[at];
  else {
    float x, unused;
    unpack2<TYPE>(((const uint16_t*)p)[at], x, unused);
    return x;
  }
}

// The number of accepted drafts, the same in every lane of a wave.
template <int TYPE>
__device__ __forceinline__ int accepted_drafts(const herschel_verify_args& a, int64_t b, int& n, bool report) {
  n = a.n_drafts;
  if (a.counts) {
    const int c = a.counts[b];
    n = max(0, min(c, a.n_drafts));
    if (report && n != c) flag(a.status, HERSCHEL_OP_BAD_LENGTH);
  }
  const int lane = threadIdx.x % WAVE;
  for (int from = 0; from < n; from += WAVE) {
    const int t = from + lane;
    bool good = false;
    if (t < n) {
      const int64_t x = a.tokens[b * a.n_drafts + t];
      const bool known = x >= 0 && x < a.vocab;
      const int64_t at = known ? x : 0;
      const double q = a.draft ? (double)probability<TYPE>(a.draft, b * a.draft_seq + t * a.draft_row + at) : 1.0;
      const double p = (double)probability<TYPE>(a.target, b * a.target_seq + t * a.target_row + at);
      good = known && (double)a.accept_u[b * a.n_drafts + t] * q < p;
      if (report && !known) flag(a.status, HERSCHEL_OP_BAD_TOKEN);
    }
    const uint64_t no = __ballot(!good);
    if (no) return from + __builtin_ctzll(no);
  }
  return n;
}

// Eight elements from `at` on of a row of probabilities; those from `end` on are 0.
// The load is in no branch but for a row's last, odd elements, so that several are
// under way at once.
typedef f32x4 f32x4_any __attribute__((aligned(4)));
typedef u32x4 u32x4_half __attribute__((aligned(2)));
template <int TYPE>
__device__ __forceinline__ void load_row(const void* base, int64_t row, int at, int end, float* x) {
  if (end >= 8) {
    const int64_t from = row + min(at, end - 8);
    if constexpr (TYPE == HERSCHEL_F32) {
      const f32x4 u = *(const f32x4_any*)((const float*)base + from), v = *(const f32x4_any*)((const float*)base + from + 4);
#pragma unroll
      for (int i = 0; i < 4; ++i) x[i] = u[i], x[i + 4] = v[i];
    } else {
      const u32x4 w = *(const u32x4_half*)((const uint16_t*)base + from);
#pragma unroll
      for (int i = 0; i < 4; ++i) unpack2<TYPE>(w[i], x[2 * i], x[2 * i + 1]);
    }
  }
  if (at + 8 > end) {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = 0;
    if (at < end) {
#pragma unroll
      for (int i = 0; i < 7; ++i)
        if (at + i < end) x[i] = probability<TYPE>(base, row + at + i);
    }
  }
}

// The row that a sequence's token is drawn from.
struct Row {
  int64_t target, draft;  // offsets of the rows
  int one;                // the draft's token, whose probability was 1; -1: there is none
  bool differs;           // target - draft, not the target alone
};
template <int TYPE>
__device__ __forceinline__ Row row_of(const herschel_verify_args& a, int64_t b, int n, int accepted) {
  Row r;
  r.target = b * a.target_seq + accepted * a.target_row;
  r.draft = b * a.draft_seq + accepted * a.draft_row;
  r.differs = accepted < n;
  r.one = -1;
  if (r.differs && !a.draft) {
    const int64_t x = a.tokens[b * a.n_drafts + accepted];
    if (x >= 0 && x < a.vocab) r.one = (int)x;
  }
  return r;
}
struct Eight {
  float p[8], q[8];
};
template <int TYPE>
__device__ __forceinline__ void load_eight(const herschel_verify_args& a, const Row& r, int at, int end, Eight& x) {
  load_row<TYPE>(a.target, r.target, at, end, x.p);
  if (r.differs && a.draft) load_row<TYPE>(a.draft, r.draft, at, end, x.q);
}
// What eight elements weigh, target - draft where that is above 0 or the target alone, and their sum.
__device__ __forceinline__ double weigh(const herschel_verify_args& a, const Row& r, int at, const Eight& x, double* w) {
  double sum = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    double d = (double)x.p[i];
    if (r.differs) d -= a.draft ? (double)x.q[i] : at + i == r.one ? 1.0 : 0.0;
    w[i] = fmax(d, 0.0);  // 0 for a NaN
    sum += w[i];
  }
  return sum;
}

__device__ __forceinline__ double wave_sum(double v) {
#pragma unroll
  for (int o = 1; o < WAVE; o *= 2) v += __shfl_xor(v, o);
  return v;
}

// What a share weighs.
template <int TYPE>
__global__ __launch_bounds__(VERIFY_THREADS) void k_verify_sums(VerifyArgs p) {
  const herschel_verify_args& a = p.a;
  __shared__ double box[VERIFY_WAVES];
  const int64_t b = blockIdx.y;
  int n;
  const int accepted = accepted_drafts<TYPE>(a, b, n, blockIdx.x == 0 && threadIdx.x < WAVE);
  const Row r = row_of<TYPE>(a, b, n, accepted);
  double s = 0;
  const int from = blockIdx.x * p.size, end = min(a.vocab, from + p.size);
  for (int at = from + (int)threadIdx.x * 8; at < end; at += SHARE_STEP) {
    Eight x;
    double w[8];
    load_eight<TYPE>(a, r, at, end, x);
    s += weigh(a, r, at, x, w);
  }
  s = wave_sum(s);
  if (threadIdx.x % WAVE == 0) box[threadIdx.x / WAVE] = s;
  __syncthreads();
  if (threadIdx.x == 0) {
    s = 0;
    for (int i = 0; i < VERIFY_WAVES; ++i) s += box[i];
    ((double*)a.workspace)[b * p.shares + blockIdx.x] = s;
    if (blockIdx.x == 0) {
      int* counted = (int*)((double*)a.workspace + (int64_t)a.n_seqs * p.shares) + b * 2;
      counted[0] = accepted;
      counted[1] = n;
    }
  }
}

// The first of a wave's lanes, in order, up to which the sum of the lanes' values
// behind `base` is above `than`; without one, the last with a value above 0, or -1.
// `before`: the sum before it.
__device__ __forceinline__ int pick_lane(double v, double base, double than, double& before) {
  const int lane = threadIdx.x % WAVE;
  double up = v;
#pragma unroll
  for (int o = 1; o < WAVE; o *= 2) {
    const double below = __shfl_up(up, o);
    if (lane >= o) up += below;
  }
  const uint64_t some = __ballot(v > 0), above = __ballot(v > 0 && base + up > than);
  if (!some) return -1;
  const int at = above ? __builtin_ctzll(above) : 63 - __builtin_clzll(some);
  before = __shfl(base + up - v, at);
  return at;
}

// Draws from a row between two of its elements, as whole steps of a workgroup: each
// wave's run of it is summed, the run found in which the sum behind `base` passes
// `than` (u times the whole, with WHOLE), in it the step, the lane and the token,
// which its lane writes.  False if nothing weighs anything.
template <int TYPE, int WAVES, int KEPT, bool WHOLE>
__device__ __forceinline__ bool draw_from(const herschel_verify_args& a, const Row& r, int from, int end, double base, double than,
                                          double u, double* sums, int64_t* out) {
  constexpr int STEP = WAVES * WAVE * 8;
  const int lane = threadIdx.x % WAVE, wave = threadIdx.x / WAVE;
  const int steps = (end - from + STEP - 1) / STEP, begin = from + wave * steps * (WAVE * 8) + lane * 8;
  // rows of no more steps than these are read at once, and their sums kept
  double s[KEPT], w[8], sum = 0;
  if (steps <= KEPT) {
    Eight x[KEPT];
#pragma unroll
    for (int i = 0; i < KEPT; ++i)
      if (i < steps) load_eight<TYPE>(a, r, begin + i * (WAVE * 8), end, x[i]);
#pragma unroll
    for (int i = 0; i < KEPT; ++i) {
      s[i] = i < steps ? weigh(a, r, begin + i * (WAVE * 8), x[i], w) : 0.0;
      sum += s[i];
    }
  } else {
    for (int i = 0; i < steps; ++i) {
      Eight x;
      load_eight<TYPE>(a, r, begin + i * (WAVE * 8), end, x);
      sum += weigh(a, r, begin + i * (WAVE * 8), x, w);
    }
  }
  sum = wave_sum(sum);
  __syncthreads();  // what was in sums has been read
  if (lane == 0) sums[wave] = sum;
  __syncthreads();
  const double of_wave = lane < WAVES ? sums[lane] : 0.0;
  if constexpr (WHOLE) than = u * wave_sum(of_wave);
  double before = 0;
  const int at = pick_lane(of_wave, base, than, before);
  if (at < 0) return false;
  if (wave != at) return true;
  int step = -1;
  double up = before, of_lane = 0;
  for (int i = 0; i < steps; ++i) {
    double v = 0;
    if (steps <= KEPT) {
#pragma unroll
      for (int k = 0; k < KEPT; ++k)
        if (k == i) v = s[k];
    } else {
      Eight x;
      load_eight<TYPE>(a, r, begin + i * (WAVE * 8), end, x);
      v = weigh(a, r, begin + i * (WAVE * 8), x, w);
    }
    const double all = wave_sum(v);
    if (!(all > 0)) continue;
    step = i;
    of_lane = v;
    before = up;
    up += all;
    if (up > than) break;
  }
  if (lane != pick_lane(of_lane, before, than, up)) return true;
  Eight x;
  const int first = begin + step * (WAVE * 8);
  load_eight<TYPE>(a, r, first, end, x);
  weigh(a, r, first, x, w);
  int token = -1;
  bool above = false;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    if (above || !(w[e] > 0)) continue;
    token = first + e;
    up += w[e];
    above = up > than;
  }
  *out = token;
  return true;
}

// The token of each sequence, and the outputs.
template <int TYPE, int THREADS, bool ONE>
__global__ __launch_bounds__(THREADS) void k_verify_draw(VerifyArgs p) {
  constexpr int WAVES = THREADS / WAVE;
  const herschel_verify_args& a = p.a;
  __shared__ double sums[WAVES];
  const int64_t b = blockIdx.x;
  const int tid = threadIdx.x, lane = tid % WAVE;
  const double u = (double)a.final_u[b];
  int n, accepted;
  if constexpr (ONE) {
    accepted = accepted_drafts<TYPE>(a, b, n, tid < WAVE);
  } else {
    const int* counted = (const int*)((const double*)a.workspace + (int64_t)a.n_seqs * p.shares) + b * 2;
    accepted = counted[0];
    n = counted[1];
  }
  Row r = row_of<TYPE>(a, b, n, accepted);
  int64_t* const out = a.out + b * (a.n_drafts + 1);
  for (int t = tid; t <= a.n_drafts; t += THREADS)
    if (t != accepted) out[t] = t < accepted ? a.tokens[b * a.n_drafts + t] : -1;
  if (tid == 0) a.accepted[b] = accepted;

  bool drawn = false;
  if constexpr (ONE) {
    drawn = draw_from<TYPE, WAVES, 4, true>(a, r, 0, a.vocab, 0.0, 0.0, u, sums, out + accepted);
  } else {
    // the share, each wave by itself; a run of shares a lane
    const double* of = (const double*)a.workspace + b * p.shares;
    const int run = (p.shares + WAVE - 1) / WAVE, first = lane * run, last = min(p.shares, first + run);
    double v = 0, base = 0;
    for (int i = first; i < last; ++i) v += of[i];
    const double than = u * wave_sum(v);
    const int at = pick_lane(v, 0.0, than, base);
    if (at >= 0) {
      int share = -1;
      for (int i = at * run; i < min(p.shares, at * run + run); ++i) {  // the same in every lane
        const double w = of[i];
        if (!(w > 0)) continue;
        if (share >= 0) base += of[share];
        share = i;
        if (base + w > than) break;
      }
      drawn = draw_from<TYPE, WAVES, 2, false>(a, r, share * p.size, min(a.vocab, (share + 1) * p.size), base, than, u, sums,
                                               out + accepted);
    }
  }
  if (drawn) return;
  // nothing of the target is above the draft: the target alone
  if (r.differs) {
    r.differs = false;
    drawn = draw_from<TYPE, WAVES, 1, true>(a, r, 0, a.vocab, 0.0, 0.0, u, sums, out + accepted);
  }
  if (!drawn && tid == 0) {
    out[accepted] = -1;
    flag(a.status, HERSCHEL_OP_BAD_ROW);
  }
}

inline int shares_of(int vocab, int n_seqs, int& size) {
  size = SHARE_STEP;
  while (size < MOST_STEPS * SHARE_STEP && (int64_t)((vocab + size - 1) / size) * n_seqs > 4096) size *= 2;
  return (vocab + size - 1) / size;
}

}  // namespace hop

extern "C" int herschel_verify_workspace(int32_t n_seqs, int32_t vocab, size_t* bytes) {
  using namespace hop;
  if (!bytes || n_seqs < 0 || n_seqs > 65535 || vocab < 1 || vocab > 0x40000000) return HERSCHEL_EINVAL;
  int size;
  *bytes = vocab <= ONE_ROW ? 0 : (size_t)n_seqs * (shares_of(vocab, n_seqs, size) * sizeof(double) + 2 * sizeof(int));
  return HERSCHEL_OK;
}

extern "C" int herschel_verify_drafts(const herschel_verify_args* args) {
  using namespace hop;
  if (!args) return HERSCHEL_EINVAL;
  const herschel_verify_args& a = *args;
  size_t need = 0;
  if (herschel_verify_workspace(a.n_seqs, a.vocab, &need) != HERSCHEL_OK) return HERSCHEL_EINVAL;
  if (a.n_drafts < 0 || a.n_drafts > HERSCHEL_MAX_DRAFTS) return HERSCHEL_EINVAL;
  if (a.type != HERSCHEL_F32 && !type_ok(a.type)) return HERSCHEL_EINVAL;
  if (a.target_seq < 0 || a.target_row < 0 || a.draft_seq < 0 || a.draft_row < 0) return HERSCHEL_EINVAL;
  if (a.n_seqs == 0) return HERSCHEL_OK;  // nothing to point at
  const size_t to = a.type == HERSCHEL_F32 ? 4 : 2;
  if (!a.target || !aligned(a.target, to) || !aligned(a.draft, to) || !a.final_u || !a.out || !a.accepted)
    return HERSCHEL_EINVAL;
  if (a.n_drafts && (!a.tokens || !a.accept_u)) return HERSCHEL_EINVAL;
  if (need && (a.workspace_bytes < need || !a.workspace || !aligned(a.workspace, 16))) return HERSCHEL_EWORKSPACE;
  // a sequence's workgroup reads its tokens, and others theirs, while some have written
  const int64_t seqs = a.n_seqs, drafts = a.n_drafts;
  const RowsMemory written[3] = {{a.out, 1, 0, seqs * (drafts + 1) * 8}, {a.accepted, 1, 0, seqs * 4}, {a.workspace, 1, 0, (int64_t)need}};
  const RowsMemory read[4] = {{drafts ? a.tokens : nullptr, 1, 0, seqs * drafts * 8}, {a.counts, 1, 0, seqs * 4},
                              {drafts ? a.accept_u : nullptr, 1, 0, seqs * drafts * 4}, {a.final_u, 1, 0, seqs * 4}};
  auto probabilities = [&](const RowsMemory& w, const void* from, int64_t seq, int64_t row, int64_t rows) {
    if (!from || !share_memory(w, {from, 1, 0, ((seqs - 1) * seq + (rows - 1) * row + a.vocab) * (int64_t)to})) return false;
    for (int64_t t = 0; t < rows; ++t)
      if (share_memory(w, {(const char*)from + t * row * (int64_t)to, seqs, seq * (int64_t)to, a.vocab * (int64_t)to})) return true;
    return false;
  };
  for (int i = 0; i < 3; ++i) {
    for (const RowsMemory& r : read)
      if (share_memory(written[i], r)) return HERSCHEL_EINVAL;
    if (probabilities(written[i], a.target, a.target_seq, a.target_row, drafts + 1)) return HERSCHEL_EINVAL;
    if (probabilities(written[i], a.draft, a.draft_seq, a.draft_row, drafts)) return HERSCHEL_EINVAL;
    for (int j = 0; j < i; ++j)
      if (share_memory(written[i], written[j])) return HERSCHEL_EINVAL;
  }
  VerifyArgs p{a};
  p.shares = shares_of(a.vocab, a.n_seqs, p.size);
  const bool f32 = a.type == HERSCHEL_F32, bf = a.type == HERSCHEL_BF16;
  if (!need)
    return launch(f32  ? k_verify_draw<HERSCHEL_F32, ONE_THREADS, true>
                  : bf ? k_verify_draw<HERSCHEL_BF16, ONE_THREADS, true>
                       : k_verify_draw<HERSCHEL_F16, ONE_THREADS, true>,
                  dim3((unsigned)a.n_seqs), dim3(ONE_THREADS), 0, a.hip_stream, p);
  const int code = launch(f32  ? k_verify_sums<HERSCHEL_F32>
                          : bf ? k_verify_sums<HERSCHEL_BF16>
                               : k_verify_sums<HERSCHEL_F16>,
                          dim3((unsigned)p.shares, (unsigned)a.n_seqs), dim3(VERIFY_THREADS), 0, a.hip_stream, p);
  if (code != HERSCHEL_OK) return code;
  return launch(f32  ? k_verify_draw<HERSCHEL_F32, VERIFY_THREADS, false>
                : bf ? k_verify_draw<HERSCHEL_BF16, VERIFY_THREADS, false>
                     : k_verify_draw<HERSCHEL_F16, VERIFY_THREADS, false>,
                dim3((unsigned)a.n_seqs), dim3(VERIFY_THREADS), 0, a.hip_stream, p);
}
