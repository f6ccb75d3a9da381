// The norms before and after a block, with its gate and residual scale, and their backward.
//
//   entry     n = Norm_in(h; gamma, beta)
//   exit      h' = a h + s act(gate) * m,  m = Norm_out(y; gamma, beta) or y;  n' = Norm_in(h'; ..)
//   Norm      x^ = (x - mean) / sqrt(var + eps) (LayerNorm; population variance), or
//             x / sqrt(mean x^2 + eps) (RMS); Norm = x^ gamma + beta
//   backward  with v = gamma * (gradient of Norm's output):
//             dx = (v - mean(v) - x^ mean(v x^)) / spread  (the mean(v) for LayerNorm only)
//
// Every tensor is read and written once.  A row lives in the registers of a wave, or of a workgroup
// where it is wide or rows are few, so that the row's sums, the norm, the gate, the residual sum and the
// next entry's norm need no second pass over memory; statistics are recomputed by the backward from the
// row it has to read in any case, and none are stored.
#include <algorithm>

#include "block_rows.h"

namespace umem {
namespace {

constexpr int THREADS = 256;

struct EntryArgs {
  const void* h;
  const float *gamma, *beta;
  void* n;
  int T, d;
  bool centre;
  float eps;
};

struct ExitArgs {
  const void *h, *y, *gate;
  const float *gamma, *beta, *gamma_next, *beta_next;
  void *h_out, *n_next;
  int T, d, norm_out, gate_kind;
  bool sigmoid, centre_next;
  float eps, a, s;
};

__device__ __forceinline__ float sigmoid(float z) { return 1.0f / (1.0f + expf(-z)); }

// Threads of a group: 64 (a wave, four rows a workgroup), or a workgroup of 256 or 1024.
template <int G>
struct Group {
  static constexpr int kThreads = G > THREADS ? G : THREADS;
  static constexpr int kRows = kThreads / G;
  static __device__ __forceinline__ int lane() { return threadIdx.x % G; }
  static __device__ __forceinline__ int index() { return threadIdx.x / G; }
};

template <int G, int PER, bool VEC, typename T>
__device__ __forceinline__ void affine_store(const RowRegs<PER>& x, const float* gamma, const float* beta, T* row,
                                             int lane, int d) {
#pragma unroll
  for (int p = 0; p < PER; ++p) {
    const int e = (p * G + lane) * 4;
    bf32x4 r = x.v[p] * load4<VEC>(gamma, e, d);
    if (beta != nullptr) r += load4<VEC>(beta, e, d);
    store4<VEC>(row, e, d, r);
  }
}

template <typename HT, typename YT, int G, int PER, bool VEC>
__global__ __launch_bounds__(Group<G>::kThreads) void entry_kernel(EntryArgs k) {
  __shared__ float lds[2][2][G / kWave];
  const int row = blockIdx.x * Group<G>::kRows + Group<G>::index(), lane = Group<G>::lane();
  if (row >= k.T) return;                    // whole groups: a group of several waves is a workgroup
  GroupSum<G> gs{lds, 0};
  const size_t at = static_cast<size_t>(row) * k.d;
  RowRegs<PER> x = load_row<G, PER, VEC>(static_cast<const HT*>(k.h) + at, lane, k.d);
  normalise<G>(x, lane, k.d, k.centre, k.eps, gs);
  affine_store<G, PER, VEC>(x, k.gamma, k.beta, static_cast<YT*>(k.n) + at, lane, k.d);
}

template <typename HT, typename YT, int G, int PER, bool VEC>
__global__ __launch_bounds__(Group<G>::kThreads) void exit_kernel(ExitArgs k) {
  __shared__ float lds[2][2][G / kWave];
  const int row = blockIdx.x * Group<G>::kRows + Group<G>::index(), lane = Group<G>::lane();
  if (row >= k.T) return;
  GroupSum<G> gs{lds, 0};
  const int d = k.d;
  const size_t at = static_cast<size_t>(row) * d;
  RowRegs<PER> m = load_row<G, PER, VEC>(static_cast<const YT*>(k.y) + at, lane, d);
  RowRegs<PER> h = load_row<G, PER, VEC>(static_cast<const HT*>(k.h) + at, lane, d);
  if (k.norm_out != UMEM_NORM_NONE) {
    normalise<G>(m, lane, d, k.norm_out == UMEM_NORM_LAYER, k.eps, gs);
#pragma unroll
    for (int p = 0; p < PER; ++p) {
      const int e = (p * G + lane) * 4;
      m.v[p] *= load4<VEC>(k.gamma, e, d);
      if (k.beta != nullptr) m.v[p] += load4<VEC>(k.beta, e, d);
    }
  }
  HT* h_out = static_cast<HT*>(k.h_out) + at;
  const float token = k.gate_kind == UMEM_GATE_TOKEN ? static_cast<const float*>(k.gate)[row] : 1.f;
#pragma unroll
  for (int p = 0; p < PER; ++p) {
    const int e = (p * G + lane) * 4;
    if (k.gate_kind != UMEM_GATE_NONE) {
      bf32x4 g = {token, token, token, token};
      if (k.gate_kind == UMEM_GATE_CHANNEL) g = load4<VEC>(static_cast<const float*>(k.gate), e, d);
      if (k.gate_kind == UMEM_GATE_FULL) g = load4<VEC>(static_cast<const YT*>(k.gate) + at, e, d);
      if (k.sigmoid) {
#pragma unroll
        for (int i = 0; i < 4; ++i) g[i] = sigmoid(g[i]);
      }
      m.v[p] *= g;
    }
    // the next entry's norm is taken of the stream as it is stored
#pragma unroll
    for (int i = 0; i < 4; ++i)
      h.v[p][i] = e + i < d ? static_cast<float>(static_cast<HT>(fmaf(k.a, h.v[p][i], k.s * m.v[p][i]))) : 0.f;
    store4<VEC>(h_out, e, d, h.v[p]);
  }
  if (k.n_next == nullptr) return;
  normalise<G>(h, lane, d, k.centre_next, k.eps, gs);
  affine_store<G, PER, VEC>(h, k.gamma_next, k.beta_next, static_cast<YT*>(k.n_next) + at, lane, d);
}

// ---------------------------------------------------------------- backward

struct EntryBackArgs {
  const void *h, *dn, *dres;
  const float* gamma;
  void* dh;
  float* part;                 // [workgroups][dgamma, dbeta][d]
  int T, d, groups;
  bool centre, shift;
  float eps;
};

struct ExitBackArgs {
  const void *y, *gate, *dh_out;
  const float *gamma, *beta;
  void *dh, *dy, *dgate;
  float* part;                 // [workgroups][dgamma, dbeta, dgate of a channel gate][d], those there are
  int T, d, groups, norm_out, gate_kind;
  bool sigmoid;
  float eps, a, s;
};

// A workgroup's column sums to row `q` of its partial sums: the groups' sums are added in order in LDS.
template <int G, int PER>
__device__ __forceinline__ void write_part(const RowRegs<PER>& acc, float* part, int d, int lane, float* lds) {
  constexpr int kRows = Group<G>::kRows;
#pragma unroll
  for (int p = 0; p < PER; ++p) {
    const int e = (p * G + lane) * 4;
    bf32x4 s = acc.v[p];
    if constexpr (kRows > 1) {
      __syncthreads();
      *reinterpret_cast<bf32x4*>(lds + threadIdx.x * 4) = s;
      __syncthreads();
      if (Group<G>::index() != 0) continue;
#pragma unroll
      for (int w = 1; w < kRows; ++w) s += *reinterpret_cast<const bf32x4*>(lds + (w * G + lane) * 4);
    }
    store4<false>(part, e, d, s);
  }
}

template <typename HT, typename YT, int G, int PER, bool VEC>
__global__ __launch_bounds__(Group<G>::kThreads) void entry_back_kernel(EntryBackArgs k) {
  __shared__ float lds[2][2][G / kWave];
  __shared__ __align__(16) float sums[Group<G>::kRows > 1 ? THREADS * 4 : 4];
  const int lane = Group<G>::lane(), d = k.d;
  const float inv_d = 1.0f / static_cast<float>(d);
  GroupSum<G> gs{lds, 0};
  RowRegs<PER> dg{}, db{};
  for (int row = blockIdx.x * Group<G>::kRows + Group<G>::index(); row < k.T; row += k.groups) {
    const size_t at = static_cast<size_t>(row) * d;
    RowRegs<PER> x = load_row<G, PER, VEC>(static_cast<const HT*>(k.h) + at, lane, d);
    RowRegs<PER> v = load_row<G, PER, VEC>(static_cast<const YT*>(k.dn) + at, lane, d);
    RowRegs<PER> up{};
    if (k.dres != nullptr) up = load_row<G, PER, VEC>(static_cast<const HT*>(k.dres) + at, lane, d);
    const float r = normalise<G>(x, lane, d, k.centre, k.eps, gs);
    float s0 = 0.f, s1 = 0.f;
#pragma unroll
    for (int p = 0; p < PER; ++p) {
      dg.v[p] += v.v[p] * x.v[p];
      db.v[p] += v.v[p];
      v.v[p] *= load4<VEC>(k.gamma, (p * G + lane) * 4, d);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        s0 += v.v[p][i];
        s1 = fmaf(v.v[p][i], x.v[p][i], s1);
      }
    }
    gs.sum2(s0, s1);
    s0 = k.centre ? s0 * inv_d : 0.f;
    s1 *= inv_d;
#pragma unroll
    for (int p = 0; p < PER; ++p)
      store4<VEC>(static_cast<HT*>(k.dh) + at, (p * G + lane) * 4, d, up.v[p] + (v.v[p] - s0 - x.v[p] * s1) * r);
  }
  const int q = k.shift ? 2 : 1;
  float* part = k.part + static_cast<size_t>(blockIdx.x) * q * d;
  write_part<G>(dg, part, d, lane, sums);
  if (k.shift) write_part<G>(db, part + d, d, lane, sums);
}

template <typename HT, typename YT, int G, int PER, bool VEC>
__global__ __launch_bounds__(Group<G>::kThreads) void exit_back_kernel(ExitBackArgs k) {
  __shared__ float lds[2][2][G / kWave];
  __shared__ __align__(16) float sums[Group<G>::kRows > 1 ? THREADS * 4 : 4];
  const int lane = Group<G>::lane(), d = k.d;
  const float inv_d = 1.0f / static_cast<float>(d);
  const bool norm = k.norm_out != UMEM_NORM_NONE;
  GroupSum<G> gs{lds, 0};
  RowRegs<PER> dg{}, db{}, dc{};
  for (int row = blockIdx.x * Group<G>::kRows + Group<G>::index(); row < k.T; row += k.groups) {
    const size_t at = static_cast<size_t>(row) * d;
    RowRegs<PER> x = load_row<G, PER, VEC>(static_cast<const YT*>(k.y) + at, lane, d);
    RowRegs<PER> v = load_row<G, PER, VEC>(static_cast<const HT*>(k.dh_out) + at, lane, d);
    if (k.dh != nullptr) {
#pragma unroll
      for (int p = 0; p < PER; ++p)
        store4<VEC>(static_cast<HT*>(k.dh) + at, (p * G + lane) * 4, d, v.v[p] * k.a);
    }
    float r = 1.f;
    if (norm) r = normalise<G>(x, lane, d, k.norm_out == UMEM_NORM_LAYER, k.eps, gs);
    float token = 1.f, slope_t = 1.f;
    if (k.gate_kind == UMEM_GATE_TOKEN) {
      token = static_cast<const float*>(k.gate)[row];
      if (k.sigmoid) {
        token = sigmoid(token);
        slope_t = token * (1.0f - token);
      }
    }
    float s0 = 0.f, s1 = 0.f, sg = 0.f;
#pragma unroll
    for (int p = 0; p < PER; ++p) {
      const int e = (p * G + lane) * 4;
      v.v[p] *= k.s;
      bf32x4 gamma = {1.f, 1.f, 1.f, 1.f};
      if (norm) gamma = load4<VEC>(k.gamma, e, d);
      if (k.gate_kind != UMEM_GATE_NONE) {
        bf32x4 m = x.v[p] * gamma;
        if (k.beta != nullptr) m += load4<VEC>(k.beta, e, d);
        m *= v.v[p];                                    // the gradient of the gate's value
        bf32x4 g = {token, token, token, token};
        if (k.gate_kind == UMEM_GATE_TOKEN) {
          sg += (m.x + m.y) + (m.z + m.w);
        } else {
          g = k.gate_kind == UMEM_GATE_CHANNEL ? load4<VEC>(static_cast<const float*>(k.gate), e, d)
                                               : load4<VEC>(static_cast<const YT*>(k.gate) + at, e, d);
          if (k.sigmoid) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              g[i] = sigmoid(g[i]);
              m[i] *= g[i] * (1.0f - g[i]);
            }
          }
          if (k.gate_kind == UMEM_GATE_CHANNEL) dc.v[p] += m;
          else store4<VEC>(static_cast<YT*>(k.dgate) + at, e, d, m);
        }
        v.v[p] *= g;
      }
      if (norm) {
        dg.v[p] += v.v[p] * x.v[p];
        db.v[p] += v.v[p];
        v.v[p] *= gamma;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          s0 += v.v[p][i];
          s1 = fmaf(v.v[p][i], x.v[p][i], s1);
        }
      }
    }
    if (k.gate_kind == UMEM_GATE_TOKEN) {
      sg = gs.sum(sg);
      if (lane == 0) static_cast<float*>(k.dgate)[row] = sg * slope_t;
    }
    if (norm) {
      gs.sum2(s0, s1);
      s0 = k.norm_out == UMEM_NORM_LAYER ? s0 * inv_d : 0.f;
      s1 *= inv_d;
    }
#pragma unroll
    for (int p = 0; p < PER; ++p) {
      const bf32x4 dy = norm ? (v.v[p] - s0 - x.v[p] * s1) * r : v.v[p];
      store4<VEC>(static_cast<YT*>(k.dy) + at, (p * G + lane) * 4, d, dy);
    }
  }
  const int q = (norm ? 1 : 0) + (k.beta != nullptr ? 1 : 0) + (k.gate_kind == UMEM_GATE_CHANNEL ? 1 : 0);
  if (q == 0) return;
  float* part = k.part + static_cast<size_t>(blockIdx.x) * q * d;
  if (norm) {
    write_part<G>(dg, part, d, lane, sums);
    part += d;
  }
  if (k.beta != nullptr) {
    write_part<G>(db, part, d, lane, sums);
    part += d;
  }
  if (k.gate_kind == UMEM_GATE_CHANNEL) write_part<G>(dc, part, d, lane, sums);
}

// Column c of the gradients: its partial sums added in order, by 16 threads a column and those in
// order again, so that the result does not depend on timing.  A channel gate's sum is the gradient of
// the gate's value's argument already (the slope is in every term).
struct ColumnArgs {
  const float* part;
  float* out[3];
  int q, d, parts;
  bool accumulate;
};

constexpr int kColThreads = 1024, kColWide = 64;
__global__ __launch_bounds__(kColThreads) void column_sum_kernel(ColumnArgs k) {
  __shared__ float lds[kColThreads];
  constexpr int kDeep = kColThreads / kColWide;
  const int c = blockIdx.x * kColWide + threadIdx.x % kColWide, deep = threadIdx.x / kColWide;
  const int n = k.q * k.d;
  float s = 0.f;
  if (c < n)
    for (int w = deep; w < k.parts; w += kDeep) s += k.part[static_cast<size_t>(w) * n + c];
  lds[threadIdx.x] = s;
  __syncthreads();
  if (deep != 0 || c >= n) return;
#pragma unroll
  for (int w = 1; w < kDeep; ++w) s += lds[w * kColWide + threadIdx.x];
  const int which = c / k.d;
  float* out = (which == 0 ? k.out[0] : which == 1 ? k.out[1] : k.out[2]) + (c - which * k.d);
  *out = k.accumulate ? *out + s : s;
}

// ---------------------------------------------------------------- which kernel takes which rows

constexpr int kFewRows = 1024;       // below: a workgroup a row, so that few rows still use the chip
constexpr int kMaxParts = 512;       // workgroups of a backward, and its rows of partial sums

struct Shape {
  int group, per;
};
Shape row_shape(int d, int T) {
  if (d <= 512) return {64, 2};
  if (d <= 2048 && T >= kFewRows) return {64, d <= 1024 ? 4 : 8};
  if (d <= 4096) return {256, d <= 2048 ? 2 : 4};
  return {1024, 4};
}

int back_workgroups(int d, int T) {
  const Shape s = row_shape(d, T);
  const int rows = s.group == 64 ? THREADS / 64 : 1;
  return std::min((T + rows - 1) / rows, kMaxParts);
}

bool four(const void* p, int dtype) {
  return reinterpret_cast<uintptr_t>(p) % (dtype == UMEM_BF16 ? 8 : 16) == 0;
}

}  // namespace

// One of the instances of a kernel for the types of h and y, the group and the load width.
#define UMEM_BLOCK_SHAPE(KERNEL, HT, YT, VEC)                                                              \
  if (shape.group == 64 && shape.per == 2) UMEM_BLOCK_GO((KERNEL<HT, YT, 64, 2, VEC>), 4, THREADS);         \
  else if (shape.group == 64 && shape.per == 4) UMEM_BLOCK_GO((KERNEL<HT, YT, 64, 4, VEC>), 4, THREADS);    \
  else if (shape.group == 64) UMEM_BLOCK_GO((KERNEL<HT, YT, 64, 8, VEC>), 4, THREADS);                      \
  else if (shape.group == 256 && shape.per == 2) UMEM_BLOCK_GO((KERNEL<HT, YT, 256, 2, VEC>), 1, THREADS);  \
  else if (shape.group == 256) UMEM_BLOCK_GO((KERNEL<HT, YT, 256, 4, VEC>), 1, THREADS);                    \
  else UMEM_BLOCK_GO((KERNEL<HT, YT, 1024, 4, VEC>), 1, 1024);
#define UMEM_BLOCK_VEC(KERNEL, HT, YT)               \
  if (vec) {                                         \
    UMEM_BLOCK_SHAPE(KERNEL, HT, YT, true)           \
  } else {                                           \
    UMEM_BLOCK_SHAPE(KERNEL, HT, YT, false)          \
  }
#define UMEM_BLOCK_LAUNCH(KERNEL)                                       \
  if (bd.htype == UMEM_F32 && bd.ytype == UMEM_F32) {                   \
    UMEM_BLOCK_VEC(KERNEL, float, float)                                \
  } else if (bd.htype == UMEM_F32) {                                    \
    UMEM_BLOCK_VEC(KERNEL, float, __bf16)                               \
  } else if (bd.ytype == UMEM_F32) {                                    \
    UMEM_BLOCK_VEC(KERNEL, __bf16, float)                               \
  } else {                                                              \
    UMEM_BLOCK_VEC(KERNEL, __bf16, __bf16)                              \
  }

hipError_t launch_block_in(const umem_block_desc& bd, int T, const void* h, const float* gamma, const float* beta,
                           void* n, hipStream_t s) {
  clear_stale_error();
  const EntryArgs k{h, gamma, beta, n, T, bd.d, bd.norm_in == UMEM_NORM_LAYER, bd.eps};
  const Shape shape = row_shape(bd.d, T);
  const bool vec = bd.d % 4 == 0 && four(h, bd.htype) && four(n, bd.ytype) && four(gamma, UMEM_F32) &&
                   four(beta, UMEM_F32);
#define UMEM_BLOCK_GO(K, ROWS, THR) \
  hipLaunchKernelGGL(K, dim3((T + ROWS - 1) / ROWS), dim3(THR), 0, s, k)
  UMEM_BLOCK_LAUNCH(entry_kernel)
  return hipGetLastError();
}

hipError_t launch_block_out(const umem_block_desc& bd, int T, const void* h, const void* y, const void* gate,
                            const float* gamma, const float* beta, void* h_out, const float* gamma_next,
                            const float* beta_next, void* n_next, hipStream_t s) {
  clear_stale_error();
  const ExitArgs k{h, y, gate, gamma, beta, gamma_next, beta_next, h_out, n_next, T, bd.d, bd.norm_out, bd.gate,
                   bd.gate_act == UMEM_ACT_SIGMOID, bd.norm_in == UMEM_NORM_LAYER, bd.eps, bd.res_scale,
                   bd.out_scale};
  const Shape shape = row_shape(bd.d, T);
  const bool vec = bd.d % 4 == 0 && four(h, bd.htype) && four(h_out, bd.htype) && four(y, bd.ytype) &&
                   four(n_next, bd.ytype) && four(gamma, UMEM_F32) && four(beta, UMEM_F32) &&
                   four(gamma_next, UMEM_F32) && four(beta_next, UMEM_F32) &&
                   (bd.gate == UMEM_GATE_FULL ? four(gate, bd.ytype)
                                              : bd.gate != UMEM_GATE_CHANNEL || four(gate, UMEM_F32));
  UMEM_BLOCK_LAUNCH(exit_kernel)
#undef UMEM_BLOCK_GO
  return hipGetLastError();
}

size_t block_backward_workspace_bytes(const umem_block_desc& bd, int T) {
  if (T == 0) return 0;
  const size_t bytes = static_cast<size_t>(back_workgroups(bd.d, T)) * 3 * bd.d * sizeof(float);
  return (bytes + 255) / 256 * 256;
}

namespace {

hipError_t launch_columns(const ColumnArgs& c, hipStream_t s) {
  const int n = c.q * c.d;
  hipLaunchKernelGGL(column_sum_kernel, dim3((n + kColWide - 1) / kColWide), dim3(kColThreads), 0, s, c);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_block_in_backward(const umem_block_desc& bd, int T, const void* h, const float* gamma,
                                    const void* dn, const void* dres, void* dh, float* dgamma, float* dbeta,
                                    bool accumulate, void* ws, hipStream_t s) {
  clear_stale_error();
  const Shape shape = row_shape(bd.d, T);
  const int groups = back_workgroups(bd.d, T);
  EntryBackArgs k{h, dn, dres, gamma, dh, static_cast<float*>(ws), T, bd.d,
                  groups * (shape.group == 64 ? THREADS / 64 : 1), bd.norm_in == UMEM_NORM_LAYER, dbeta != nullptr,
                  bd.eps};
  const bool vec = bd.d % 4 == 0 && four(h, bd.htype) && four(dn, bd.ytype) && four(dres, bd.htype) &&
                   four(dh, bd.htype) && four(gamma, UMEM_F32);
#define UMEM_BLOCK_GO(K, ROWS, THR) hipLaunchKernelGGL(K, dim3(groups), dim3(THR), 0, s, k)
  UMEM_BLOCK_LAUNCH(entry_back_kernel)
  hipError_t e = hipGetLastError();
  if (e == hipSuccess)
    e = launch_columns({static_cast<const float*>(ws), {dgamma, dbeta, nullptr}, dbeta ? 2 : 1, bd.d, groups, accumulate}, s);
  return e;
}

hipError_t launch_block_out_backward(const umem_block_desc& bd, int T, const void* y, const void* gate,
                                     const float* gamma, const float* beta, const void* dh_out, void* dh, void* dy,
                                     void* dgate, float* dgamma, float* dbeta, bool accumulate, void* ws,
                                     hipStream_t s) {
  clear_stale_error();
  const Shape shape = row_shape(bd.d, T);
  const int groups = back_workgroups(bd.d, T);
  ExitBackArgs k{y, gate, dh_out, gamma, beta, dh, dy, dgate, static_cast<float*>(ws), T, bd.d,
                 groups * (shape.group == 64 ? THREADS / 64 : 1), bd.norm_out, bd.gate,
                 bd.gate_act == UMEM_ACT_SIGMOID, bd.eps, bd.res_scale, bd.out_scale};
  const bool full = bd.gate == UMEM_GATE_FULL;
  const bool vec = bd.d % 4 == 0 && four(y, bd.ytype) && four(dh_out, bd.htype) && four(dh, bd.htype) &&
                   four(dy, bd.ytype) && four(gamma, UMEM_F32) && four(beta, UMEM_F32) &&
                   (full ? four(gate, bd.ytype) && four(dgate, bd.ytype)
                         : bd.gate != UMEM_GATE_CHANNEL || four(gate, UMEM_F32));
  UMEM_BLOCK_LAUNCH(exit_back_kernel)
#undef UMEM_BLOCK_GO
  hipError_t e = hipGetLastError();
  ColumnArgs c{static_cast<const float*>(ws), {nullptr, nullptr, nullptr}, 0, bd.d, groups, accumulate};
  if (dgamma != nullptr) c.out[c.q++] = dgamma;
  if (dbeta != nullptr) c.out[c.q++] = dbeta;
  if (bd.gate == UMEM_GATE_CHANNEL) c.out[c.q++] = static_cast<float*>(dgate);
  if (e == hipSuccess && c.q > 0) e = launch_columns(c, s);
  return e;
}

}  // namespace umem
