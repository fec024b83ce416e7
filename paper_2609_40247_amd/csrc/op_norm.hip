// Root-mean-square norm with the residual's addition, one launch.
//
// h = x + residual; y = h / sqrt(mean h^2 + eps) * weight, to 16 bits or to
// 8-bit codes with a scale a row or a group of columns.  A row is read once and
// stays in the registers of its workgroup: the traffic is the floor, each
// input read and each output written once, and bounds it: 8192 rows of 5120 in
// bf16 with the residual, 336 MB, 60.7 us, 5.5 TB/s.  One row of 4096 takes 2.6 us, a
// launch's latency.
#include "ops.hpp"

namespace hop {

struct NormArgs {
  herschel_norm_args a;
};

// Past the caches with STREAM.
template <bool STREAM, class T>
__device__ __forceinline__ void put(T* to, T x) {
  if constexpr (STREAM) __builtin_nontemporal_store(x, to);
  else *to = x;
}

constexpr int NORM_WAVES = 16;
constexpr int NORM_GRID = 1 << 20;  // rows of a line of workgroups: a launch's threads are counted in 32 bits

// Sum, or largest, over a workgroup of whole waves, the same in every lane; `box` is used by one call only.
__device__ __forceinline__ float block_sum(float v, float* box) {
#pragma unroll
  for (int o = 1; o < WAVE; o *= 2) v += __shfl_xor(v, o);
  const int waves = blockDim.x / WAVE;
  if (waves == 1) return v;
  if (threadIdx.x % WAVE == 0) box[threadIdx.x / WAVE] = v;
  __syncthreads();
  float s = 0;
  for (int i = 0; i < waves; ++i) s += box[i];
  return s;
}
__device__ __forceinline__ uint32_t block_max(uint32_t v, uint32_t* box) {
#pragma unroll
  for (int o = 1; o < WAVE; o *= 2) v = max(v, (uint32_t)__shfl_xor((int)v, o));
  const int waves = blockDim.x / WAVE;
  if (waves == 1) return v;
  if (threadIdx.x % WAVE == 0) box[threadIdx.x / WAVE] = v;
  __syncthreads();
  uint32_t m = 0;
  for (int i = 0; i < waves; ++i) m = max(m, box[i]);
  return m;
}

// Eight elements of a row as floats: contiguous ones (VEC), or T apart.
template <int TYPE, bool VEC>
__device__ __forceinline__ void load8(const void* base, int64_t row, int at, int T, int dim, float* x) {
  if constexpr (TYPE == HERSCHEL_F32) {
    const float* p = (const float*)base + row;
    if constexpr (VEC) {
      const f32x4 a = *(const f32x4*)(p + at), b = *(const f32x4*)(p + at + 4);
#pragma unroll
      for (int i = 0; i < 4; ++i) x[i] = a[i], x[i + 4] = b[i];
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = at + i * T < dim ? p[at + i * T] : 0.0f;
    }
  } else {
    const uint16_t* p = (const uint16_t*)base + row;
    if constexpr (VEC) {
      const u32x4 w = *(const u32x4*)(p + at);
#pragma unroll
      for (int i = 0; i < 4; ++i) unpack2<TYPE>(w[i], x[2 * i], x[2 * i + 1]);
    } else {
      float unused;
#pragma unroll
      for (int i = 0; i < 8; ++i) unpack2<TYPE>(at + i * T < dim ? p[at + i * T] : (uint16_t)0, x[i], unused);
    }
  }
}
template <int TYPE, bool VEC, bool STREAM>
__device__ __forceinline__ void store8(void* base, int64_t row, int at, int T, int dim, const float* x) {
  if constexpr (TYPE == HERSCHEL_F32) {
    float* p = (float*)base + row;
    if constexpr (VEC) {
      put<STREAM>((f32x4*)(p + at), f32x4{x[0], x[1], x[2], x[3]});
      put<STREAM>((f32x4*)(p + at + 4), f32x4{x[4], x[5], x[6], x[7]});
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (at + i * T < dim) p[at + i * T] = x[i];
    }
  } else {
    uint16_t* p = (uint16_t*)base + row;
    if constexpr (VEC) {
      u32x4 w;
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] = pack2<TYPE>(x[2 * i], x[2 * i + 1]);
      put<STREAM>((u32x4*)(p + at), w);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (at + i * T < dim) p[at + i * T] = (uint16_t)pack2<TYPE>(x[i], 0.0f);
    }
  }
}

// A workgroup to a row, V times eight elements a thread.  VEC: eight neighbours
// each, for rows of whole 16-byte chunks; else elements a workgroup apart.
template <int TYPE, int OUT, int V, bool VEC, bool STREAM>
__global__ __launch_bounds__(1024) void k_norm(NormArgs p) {
  const herschel_norm_args& a = p.a;
  __shared__ float box[NORM_WAVES], box2[NORM_WAVES];
  __shared__ uint32_t top[NORM_WAVES], top2[NORM_WAVES];
  __shared__ uint32_t of_group[VEC || !quantised(OUT) ? 1 : HERSCHEL_MAX_NORM_DIM / 32];
  const int T = blockDim.x, tid = threadIdx.x, dim = a.dim;
  const int64_t row = (int64_t)blockIdx.y * NORM_GRID + blockIdx.x;
  if (row >= a.n_rows) return;
  int at[V];
  bool has[V];
  float h[V][8], w[V][8];
#pragma unroll
  for (int v = 0; v < V; ++v) {
    at[v] = VEC ? (v * T + tid) * 8 : v * T * 8 + tid;
    has[v] = at[v] < dim;
#pragma unroll
    for (int i = 0; i < 8; ++i) h[v][i] = w[v][i] = 0;
    if (has[v]) load8<TYPE, VEC>(a.x, row * a.x_row, at[v], T, dim, h[v]);
  }
  if (a.residual) {
    float r[V][8];
#pragma unroll
    for (int v = 0; v < V; ++v) {
      if (!has[v]) continue;
      if (a.residual_type == HERSCHEL_F32) load8<HERSCHEL_F32, VEC>(a.residual, row * a.residual_row, at[v], T, dim, r[v]);
      else load8<TYPE, VEC>(a.residual, row * a.residual_row, at[v], T, dim, r[v]);
    }
#pragma unroll
    for (int v = 0; v < V; ++v)
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (has[v]) h[v][i] += r[v][i];
  }
#pragma unroll
  for (int v = 0; v < V; ++v) {
    if (!has[v]) continue;
    if (a.weight_type == HERSCHEL_F32) load8<HERSCHEL_F32, VEC>(a.weight, 0, at[v], T, dim, w[v]);
    else load8<TYPE, VEC>(a.weight, 0, at[v], T, dim, w[v]);
  }
  if (a.residual_out) {
#pragma unroll
    for (int v = 0; v < V; ++v) {
      if (!has[v]) continue;
      if (a.residual_type == HERSCHEL_F32)
        store8<HERSCHEL_F32, VEC, STREAM>(a.residual_out, row * a.residual_out_row, at[v], T, dim, h[v]);
      else store8<TYPE, VEC, STREAM>(a.residual_out, row * a.residual_out_row, at[v], T, dim, h[v]);
    }
  }
  float s = 0;
#pragma unroll
  for (int v = 0; v < V; ++v)
#pragma unroll
    for (int i = 0; i < 8; ++i) s += h[v][i] * h[v][i];
  s = block_sum(s, box);
  float eps = a.eps;
  // Squares that may have left 32 bits, above or below: again, of the row times the power of two that its
  // largest magnitude calls for.  Below only where eps does not outweigh them.
  if (!(s < 0x1p100f) || (s < 0x1p-80f && eps < 0x1p-80f)) {
    uint32_t m = 0;
#pragma unroll
    for (int v = 0; v < V; ++v)
#pragma unroll
      for (int i = 0; i < 8; ++i) m = max(m, __builtin_bit_cast(uint32_t, h[v][i]) & 0x7fffffffu);
    m = block_max(m, top);
    const int e = __builtin_amdgcn_frexp_expf(__builtin_bit_cast(float, m));
    const float k = ldexpf(eps, -2 * e);
    if (m != 0 && m < 0x7f800000u && k < INFINITY) {
      eps = k;
      s = 0;
#pragma unroll
      for (int v = 0; v < V; ++v)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          h[v][i] = ldexpf(h[v][i], -e);
          s += h[v][i] * h[v][i];
        }
      s = block_sum(s, box2);
    }
  }
  const float by = 1.0f / sqrtf(s / (float)dim + eps);
#pragma unroll
  for (int v = 0; v < V; ++v)
#pragma unroll
    for (int i = 0; i < 8; ++i) h[v][i] = h[v][i] * by * w[v][i];
  if constexpr (!quantised(OUT)) {
#pragma unroll
    for (int v = 0; v < V; ++v)
      if (has[v]) store8<TYPE, VEC, STREAM>(a.out, row * dim, at[v], T, dim, h[v]);
  } else {
    // magnitudes as bits order like the numbers, with infinity and NaN above all
    uint32_t m[V], all = 0;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      m[v] = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (VEC ? has[v] : at[v] + i * T < dim) m[v] = max(m[v], __builtin_bit_cast(uint32_t, h[v][i]) & 0x7fffffffu);
      all = max(all, m[v]);
    }
    uint8_t* out = (uint8_t*)a.out + row * dim;
    const int groups = a.group ? dim / a.group : 1;
    float inv, scale;
    if (!a.group) {
      scale = row_scale<OUT>(block_max(all, top2), inv);
      if (tid == 0) a.scale[row] = scale;
    } else if constexpr (!VEC) {
      for (int g = tid; g < groups; g += T) of_group[g] = 0;
      __syncthreads();
#pragma unroll
      for (int v = 0; v < V; ++v)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int c = at[v] + i * T;
          if (c < dim) atomicMax(of_group + c / a.group, __builtin_bit_cast(uint32_t, h[v][i]) & 0x7fffffffu);
        }
      __syncthreads();
    }
#pragma unroll
    for (int v = 0; v < V; ++v) {
      if constexpr (VEC) {
        if (a.group) {  // a group's lanes are neighbours
          for (int o = 1; o < a.group / 8; o *= 2) m[v] = max(m[v], (uint32_t)__shfl_xor((int)m[v], o));
          scale = row_scale<OUT>(m[v], inv);
          if (has[v] && at[v] % a.group == 0) a.scale[row * groups + at[v] / a.group] = scale;
        }
        if (has[v]) put<STREAM>((u32x2*)(out + at[v]), u32x2{encode4<OUT>(h[v], inv), encode4<OUT>(h[v] + 4, inv)});
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int c = at[v] + i * T;
          if (c >= dim) continue;
          if (a.group) {
            scale = row_scale<OUT>(of_group[c / a.group], inv);
            if (c % a.group == 0) a.scale[row * groups + c / a.group] = scale;
          }
          const float one[4] = {h[v][i], 0, 0, 0};
          out[c] = (uint8_t)encode4<OUT>(one, inv);
        }
      }
    }
  }
}

template <int TYPE, int OUT>
static int norm_launch(NormArgs& p) {
  const herschel_norm_args& a = p.a;
  const int res = a.residual_type == HERSCHEL_F32 ? 4 : 2;
  auto rows16 = [&](const void* q, int64_t row, int bytes) { return aligned(q, 16) && row * bytes % 16 == 0; };
  const bool vec = a.dim % 8 == 0 && rows16(a.x, a.x_row, 2) && rows16(a.residual, a.residual_row, res) &&
                   rows16(a.residual_out, a.residual_out_row, res) && aligned(a.weight, 16) &&
                   aligned(a.out, quantised(OUT) ? 8 : 16);
  // What is written goes past the caches, which hold what is still to be read, where there is much of it (8192 rows of
  // 5120 66.4 to 61.0 us, 2048 of 4096 12.2 to 12.1); a step's few rows stay in them for the product that reads
  // them next.  Measured on the norm alone: what the product of a prompt's rows pays for it has not been.
  const bool stream = a.n_rows * a.dim >= (1 << 22);
  // A workgroup to a row, a thread to eight of its elements, to sixteen where there are rows enough to fill the card
  // (8192 rows of 5120 in bf16 with a residual 61.0 us against 62.9 with eight, to fp8 58.4 against 69.5; 2048 of 4096
  // 12.1 against 11.8; one row of 4096 2.6 against 3.2 with sixteen), to 32 for the longest.
  const int eights = (a.dim + 7) / 8, share = a.n_rows < 2048 ? 1 : 2;
  int V = 1, T = (eights + WAVE - 1) / WAVE * WAVE;
  while (V < 4 && (T > 1024 || (T > 256 && V < share))) {
    V *= 2;
    T = (eights + V * WAVE - 1) / (V * WAVE) * WAVE;
  }
  void (*k)(NormArgs);
  if (vec && stream)
    k = V == 1 ? k_norm<TYPE, OUT, 1, true, true> : V == 2 ? k_norm<TYPE, OUT, 2, true, true> : k_norm<TYPE, OUT, 4, true, true>;
  else if (vec)
    k = V == 1 ? k_norm<TYPE, OUT, 1, true, false> : V == 2 ? k_norm<TYPE, OUT, 2, true, false> : k_norm<TYPE, OUT, 4, true, false>;
  else
    k = V == 1 ? k_norm<TYPE, OUT, 1, false, false> : V == 2 ? k_norm<TYPE, OUT, 2, false, false> : k_norm<TYPE, OUT, 4, false, false>;
  const int64_t across = a.n_rows < NORM_GRID ? a.n_rows : NORM_GRID;
  return launch(k, dim3((unsigned)across, (unsigned)((a.n_rows + NORM_GRID - 1) / NORM_GRID)), dim3(T), 0, a.hip_stream, p);
}

template <int TYPE>
static int norm_kind(NormArgs& p) {
  switch (p.a.out_kind) {
    case HERSCHEL_FP8: return norm_launch<TYPE, HERSCHEL_FP8>(p);
    case HERSCHEL_INT8: return norm_launch<TYPE, HERSCHEL_INT8>(p);
    default: return norm_launch<TYPE, TYPE>(p);
  }
}

}  // namespace hop

extern "C" int herschel_norm_rows(const herschel_norm_args* args) {
  using namespace hop;
  if (!args) return HERSCHEL_EINVAL;
  const herschel_norm_args& a = *args;
  if (!type_ok(a.type) || a.n_rows < 0 || a.n_rows > 0x7fffffff || a.dim < 1 || a.dim > HERSCHEL_MAX_NORM_DIM)
    return HERSCHEL_EINVAL;
  if ((a.out_kind != a.type && !quantised(a.out_kind)) || (a.weight_type != a.type && a.weight_type != HERSCHEL_F32))
    return HERSCHEL_EINVAL;
  if (!(a.eps >= 0) || !(a.eps < INFINITY) || a.x_row < 0) return HERSCHEL_EINVAL;
  if (a.group && (!quantised(a.out_kind) || (a.group != 32 && a.group != 64 && a.group != 128) || a.dim % a.group))
    return HERSCHEL_EINVAL;
  if (a.residual || a.residual_out) {
    if (!a.residual && a.n_rows) return HERSCHEL_EINVAL;
    if ((a.residual_type != a.type && a.residual_type != HERSCHEL_F32) || a.residual_row < 0) return HERSCHEL_EINVAL;
    if (a.residual_out && a.residual_out_row < a.dim) return HERSCHEL_EINVAL;
    const size_t to = a.residual_type == HERSCHEL_F32 ? 4 : 2;
    if (!aligned(a.residual, to) || !aligned(a.residual_out, to)) return HERSCHEL_EINVAL;
  }
  if (a.n_rows == 0) return HERSCHEL_OK;  // nothing to point at
  if (!a.x || !a.weight || !a.out || !aligned(a.x, 2) || !aligned(a.weight, a.weight_type == HERSCHEL_F32 ? 4 : 2))
    return HERSCHEL_EINVAL;
  if (quantised(a.out_kind) ? !a.scale || !aligned(a.scale, 4) : !aligned(a.out, 2)) return HERSCHEL_EINVAL;
  // What is written is read by no other row's workgroup: it is the rows it stands for, element by element, or memory
  // of its own.
  const int64_t rows = a.n_rows, dim = a.dim, res = a.residual_type == HERSCHEL_F32 ? 4 : 2, out = quantised(a.out_kind) ? 1 : 2;
  const int64_t groups = a.group ? dim / a.group : 1;
  const RowsMemory x{a.x, rows, a.x_row * 2, dim * 2}, residual{a.residual, rows, a.residual_row * res, dim * res},
      weight{a.weight, 1, 0, dim * (a.weight_type == HERSCHEL_F32 ? 4 : 2)},
      written[3] = {{a.residual_out, rows, a.residual_out_row * res, dim * res}, {a.out, rows, dim * out, dim * out},
                    {quantised(a.out_kind) ? a.scale : nullptr, rows, groups * 4, groups * 4}};
  auto same = [&](const RowsMemory& u, const RowsMemory& v) {
    return u.at == v.at && u.width == v.width && (u.step == v.step || rows == 1);
  };
  for (int i = 0; i < 3; ++i) {
    const RowsMemory& w = written[i];
    if (!(i < 2 && same(w, x)) && share_memory(w, x)) return HERSCHEL_EINVAL;
    if (!(i < 1 && same(w, residual)) && share_memory(w, residual)) return HERSCHEL_EINVAL;
    if (share_memory(w, weight)) return HERSCHEL_EINVAL;
    for (int j = 0; j < i; ++j)
      if (share_memory(w, written[j])) return HERSCHEL_EINVAL;
  }
  NormArgs p{a};
  return a.type == HERSCHEL_BF16 ? norm_kind<HERSCHEL_BF16>(p) : norm_kind<HERSCHEL_F16>(p);
}
