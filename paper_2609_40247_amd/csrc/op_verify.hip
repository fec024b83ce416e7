// Drafted tokens against the target's probabilities: how many are accepted, and
// the token drawn behind them.  Two launches.
//
// Only one row of the vocabulary a sequence is ever read, that of the first draft
// that is not accepted (and its counterpart of the draft's probabilities): every
// workgroup finds it by itself from the drafts' own probabilities, a few
// loads, and sums its share of the row; the second kernel finds the share in
// which the cumulative sum passes the random number's and goes over it again.
#include "ops.hpp"

namespace hop {

struct VerifyArgs {
  herschel_verify_args a;
  int shares;   // of a row
  int size;     // elements of a share, a multiple of SHARE_STEP
};

constexpr int VERIFY_THREADS = 256, VERIFY_WAVES = VERIFY_THREADS / WAVE;
constexpr int SHARE_STEP = VERIFY_THREADS * 8;

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
typedef f32x4 f32x4_any __attribute__((aligned(4)));
typedef u32x4 u32x4_half __attribute__((aligned(2)));
template <int TYPE>
__device__ __forceinline__ void load_row(const void* base, int64_t row, int at, int end, float* x) {
  if (at + 8 <= end) {
    if constexpr (TYPE == HERSCHEL_F32) {
      const f32x4 u = *(const f32x4_any*)((const float*)base + row + at), v = *(const f32x4_any*)((const float*)base + row + at + 4);
#pragma unroll
      for (int i = 0; i < 4; ++i) x[i] = u[i], x[i + 4] = v[i];
    } else {
      const u32x4 w = *(const u32x4_half*)((const uint16_t*)base + row + at);
#pragma unroll
      for (int i = 0; i < 4; ++i) unpack2<TYPE>(w[i], x[2 * i], x[2 * i + 1]);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = at + i < end ? probability<TYPE>(base, row + at + i) : 0.0f;
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
// What eight elements weigh: target - draft, or (alone) the target.
template <int TYPE>
__device__ __forceinline__ void weigh(const herschel_verify_args& a, const Row& r, int at, int end, double* both,
                                      double* alone) {
  float p[8], q[8];
  load_row<TYPE>(a.target, r.target, at, end, p);
  if (r.differs && a.draft) load_row<TYPE>(a.draft, r.draft, at, end, q);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    alone[i] = p[i] > 0 ? (double)p[i] : 0.0;
    double d = (double)p[i];
    if (r.differs) d -= a.draft ? (double)q[i] : at + i == r.one ? 1.0 : 0.0;
    both[i] = d > 0 ? d : 0.0;
  }
}

__device__ __forceinline__ double wave_sum(double v) {
#pragma unroll
  for (int o = 1; o < WAVE; o *= 2) v += __shfl_xor(v, o);
  return v;
}

// A share's sums: of target - draft, and of the target.
template <int TYPE>
__global__ __launch_bounds__(VERIFY_THREADS) void k_verify_sums(VerifyArgs p) {
  const herschel_verify_args& a = p.a;
  __shared__ double box[2][VERIFY_WAVES];
  const int64_t b = blockIdx.y;
  int n;
  const int accepted = accepted_drafts<TYPE>(a, b, n, blockIdx.x == 0 && threadIdx.x < WAVE);
  const Row r = row_of<TYPE>(a, b, n, accepted);
  double s = 0, t = 0;
  const int from = blockIdx.x * p.size, end = min(a.vocab, from + p.size);
  for (int at = from + (int)threadIdx.x * 8; at < end; at += SHARE_STEP) {
    double both[8], alone[8];
    weigh<TYPE>(a, r, at, end, both, alone);
#pragma unroll
    for (int i = 0; i < 8; ++i) s += both[i], t += alone[i];
  }
  s = wave_sum(s);
  t = wave_sum(t);
  if (threadIdx.x % WAVE == 0) box[0][threadIdx.x / WAVE] = s, box[1][threadIdx.x / WAVE] = t;
  __syncthreads();
  if (threadIdx.x == 0) {
    double* out = (double*)a.workspace + (b * p.shares + blockIdx.x) * 2;
    s = t = 0;
    for (int i = 0; i < VERIFY_WAVES; ++i) s += box[0][i], t += box[1][i];
    out[0] = s;
    out[1] = t;
  }
}

// The first of a workgroup's threads, in order, behind whose v the sum of the
// values up to it is above `than`, and the sum before it; if there is none, the
// last with a value above 0; -1 if there is none either.  Returns the whole sum too.
struct Place {
  int thread;
  double before, all;
};
__device__ __forceinline__ Place place(double v, double base, double than, double* sums, int* found) {
  const int lane = threadIdx.x % WAVE, wave = threadIdx.x / WAVE;
  double up = v;
#pragma unroll
  for (int o = 1; o < WAVE; o *= 2) {
    const double below = __shfl_up(up, o);
    if (lane >= o) up += below;
  }
  __syncthreads();  // what was in sums and found has been read
  if (lane == WAVE - 1) sums[wave] = up;
  if (threadIdx.x < 2) found[threadIdx.x] = threadIdx.x == 0 ? VERIFY_THREADS : -1;
  __syncthreads();
  double before = base, all = 0;
  for (int i = 0; i < VERIFY_WAVES; ++i) {
    if (i < wave) before += sums[i];
    all += sums[i];
  }
  if (before + up > than && v > 0) atomicMin(found, (int)threadIdx.x);
  if (v > 0) atomicMax(found + 1, (int)threadIdx.x);
  __syncthreads();
  Place r;
  r.thread = found[0] < VERIFY_THREADS ? found[0] : found[1];
  r.before = before + up - v;
  r.all = all;
  return r;
}

// The token of each sequence, and the outputs.
template <int TYPE>
__global__ __launch_bounds__(VERIFY_THREADS) void k_verify_draw(VerifyArgs p) {
  const herschel_verify_args& a = p.a;
  __shared__ double sums[VERIFY_WAVES], start;
  __shared__ int found[2], token;
  const int64_t b = blockIdx.x;
  const int tid = threadIdx.x;
  int n;
  const int accepted = accepted_drafts<TYPE>(a, b, n, false);
  Row r = row_of<TYPE>(a, b, n, accepted);
  for (int t = tid; t <= a.n_drafts; t += VERIFY_THREADS)
    if (t != accepted) a.out[b * (a.n_drafts + 1) + t] = t < accepted ? a.tokens[b * a.n_drafts + t] : -1;

  // the shares' sums, a run of them a thread
  const double* of = (const double*)a.workspace + b * p.shares * 2;
  const int run = (p.shares + VERIFY_THREADS - 1) / VERIFY_THREADS, first = tid * run, last = min(p.shares, first + run);
  double both = 0, alone = 0;
  for (int i = first; i < last; ++i) both += of[2 * i], alone += of[2 * i + 1];
  Place at = place(both, 0.0, INFINITY, sums, found);
  int which = 0;
  if (!(at.all > 0)) {  // nothing of the target is above the draft: the target alone
    which = 1;
    r.differs = false;
    at = place(alone, 0.0, INFINITY, sums, found);
  }
  const double than = (double)a.final_u[b] * at.all;
  at = place(which ? alone : both, 0.0, than, sums, found);
  if (tid == 0) {
    a.accepted[b] = accepted;
    token = -1;
    if (at.thread < 0) flag(a.status, HERSCHEL_OP_BAD_ROW);
  }
  if (at.thread < 0) {
    if (tid == 0) a.out[b * (a.n_drafts + 1) + accepted] = -1;
    return;
  }
  __syncthreads();
  if (tid == at.thread) {  // the share of the run
    double s = at.before;
    int share = -1;
    for (int i = first; i < last; ++i) {
      const double v = of[2 * i + which];
      if (!(v > 0)) continue;
      share = i;
      start = s;
      s += v;
      if (s > than) break;
    }
    token = share;
  }
  __syncthreads();
  const int share = token, from = share * p.size, end = min(a.vocab, from + p.size);
  double base = start;
  // the share's elements, eight a thread
  int behind = -1;  // the last element above 0 so far
  __shared__ int pick;
  for (int at0 = from; at0 < end; at0 += SHARE_STEP) {
    double w[8], unused[8], s = 0;
    const int mine = at0 + tid * 8;
    weigh<TYPE>(a, r, mine, end, w, unused);
#pragma unroll
    for (int i = 0; i < 8; ++i) s += w[i];
    const Place e = place(s, base, than, sums, found);
    if (tid == e.thread) {
      double up = e.before;
      int k = -1;
      bool above = false;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        if (above || !(w[i] > 0)) continue;
        k = mine + i;
        up += w[i];
        above = up > than;
      }
      pick = k;
    }
    const bool done = found[0] < VERIFY_THREADS;
    __syncthreads();
    if (e.thread >= 0) behind = pick;
    base += e.all;
    if (done) break;
    __syncthreads();
  }
  if (tid == 0) a.out[b * (a.n_drafts + 1) + accepted] = behind;
}

inline int shares_of(int vocab, int n_seqs, int& size) {
  size = SHARE_STEP;
  while (size < 16 * SHARE_STEP && (int64_t)((vocab + size - 1) / size) * n_seqs > 4096) size *= 2;
  return (vocab + size - 1) / size;
}

}  // namespace hop

extern "C" int herschel_verify_workspace(int32_t n_seqs, int32_t vocab, size_t* bytes) {
  using namespace hop;
  if (!bytes || n_seqs < 0 || n_seqs > 65535 || vocab < 1 || vocab > 0x40000000) return HERSCHEL_EINVAL;
  // shares are no smaller than these
  *bytes = (size_t)n_seqs * ((vocab + SHARE_STEP - 1) / SHARE_STEP) * 2 * sizeof(double);
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
  if (a.workspace_bytes < need || !a.workspace || !aligned(a.workspace, 16)) return HERSCHEL_EWORKSPACE;
  VerifyArgs p{a};
  p.shares = shares_of(a.vocab, a.n_seqs, p.size);
  const bool f32 = a.type == HERSCHEL_F32, bf = a.type == HERSCHEL_BF16;
  const int code = launch(f32  ? k_verify_sums<HERSCHEL_F32>
                          : bf ? k_verify_sums<HERSCHEL_BF16>
                               : k_verify_sums<HERSCHEL_F16>,
                          dim3((unsigned)p.shares, (unsigned)a.n_seqs), dim3(VERIFY_THREADS), 0, a.hip_stream, p);
  if (code != HERSCHEL_OK) return code;
  return launch(f32  ? k_verify_draw<HERSCHEL_F32>
                : bf ? k_verify_draw<HERSCHEL_BF16>
                     : k_verify_draw<HERSCHEL_F16>,
                dim3((unsigned)a.n_seqs), dim3(VERIFY_THREADS), 0, a.hip_stream, p);
}
