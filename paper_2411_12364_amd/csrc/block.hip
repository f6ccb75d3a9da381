// The norms before and after a block, with its gate and residual scale.
//
//   entry     n = Norm_in(h; gamma, beta)
//   exit      h' = a h + s act(gate) * m,  m = Norm_out(y; gamma, beta) or y;  n' = Norm_in(h'; ..)
//   Norm      x^ = (x - mean) / sqrt(var + eps) (LayerNorm; population variance), or
//             x / sqrt(mean x^2 + eps) (RMS); Norm = x^ gamma + beta
//
// Bound by HBM for many rows, by the latency of one load, two to four sums and one store for few.  Every
// tensor is read and written once: a row lives in the registers of a wave or a workgroup, so the norm, the
// gate, the residual sum and the next entry's norm need no second pass over memory.  A group walks rows a
// launch's width apart with the parameters of its columns kept in registers (read again for each row they
// were as many bytes from L2 as the row from HBM), the next row's loads in flight while it sums this one.
#include "block_rows.h"

namespace umem {
namespace {

struct EntryArgs {
  const void* h;
  const float *gamma, *beta;
  void* n;
  int T, d, stride;            // rows of all groups together
  bool centre;
  float eps;
};

struct ExitArgs {
  const void *h, *y, *gate;
  const float *gamma, *beta, *gamma_next, *beta_next;
  void *h_out, *n_next;
  int T, d, stride, norm_out, gate_kind;
  bool sigmoid, centre_next;
  float eps, a, s;
};

template <int PER>
__device__ __forceinline__ Row<PER> affine(const Row<PER>& x, const Row<PER>& gamma, const Row<PER>& beta) {
  Row<PER> r;
#pragma unroll
  for (int p = 0; p < PER; ++p)
#pragma unroll
    for (int i = 0; i < 4; ++i) r.v[p][i] = fmaf(x.v[p][i], gamma.v[p][i], beta.v[p][i]);
  return r;
}

template <typename HT, typename YT, int G, int PER, RowEnd END>
__global__ __launch_bounds__(Group<G>::kThreads) void entry_kernel(EntryArgs k) {
  __shared__ float lds[2][Group<G>::kWaves][2];
  const int lane = Group<G>::lane(), d = k.d;
  int row = blockIdx.x * Group<G>::kRows + Group<G>::index();
  if (row >= k.T) return;                    // whole groups: a group of several waves is a workgroup
  GroupSum<G> gs{lds, 0};
  const HT* h = static_cast<const HT*>(k.h);
  RawRow<HT, PER> ahead = load_raw<G, PER, END>(h + static_cast<size_t>(row) * d, lane, d);
  const Row<PER> gamma = load_params<G, PER, END>(k.gamma, 1.f, lane, d), beta = load_params<G, PER, END>(k.beta, 0.f, lane, d);
  for (; row < k.T; row += k.stride) {
    Row<PER> x = widen<G, END>(ahead, lane, d);
    if (row + k.stride < k.T) ahead = load_raw<G, PER, END>(h + static_cast<size_t>(row + k.stride) * d, lane, d);
    normalise<G, END>(x, lane, d, k.centre, k.eps, gs);
    store_row<G, END>(static_cast<YT*>(k.n) + static_cast<size_t>(row) * d, affine(x, gamma, beta), lane, d);
  }
}

template <typename HT, typename YT, int G, int PER, RowEnd END>
__global__ __launch_bounds__(Group<G>::kThreads) void exit_kernel(ExitArgs k) {
  __shared__ float lds[2][Group<G>::kWaves][2];
  const int lane = Group<G>::lane(), d = k.d;
  int row = blockIdx.x * Group<G>::kRows + Group<G>::index();
  if (row >= k.T) return;
  GroupSum<G> gs{lds, 0};
  const HT* h = static_cast<const HT*>(k.h);
  const YT *y = static_cast<const YT*>(k.y), *full = static_cast<const YT*>(k.gate);
  const bool norm = k.norm_out != UMEM_NORM_NONE, gated = k.gate_kind == UMEM_GATE_FULL,
             by_channel = k.gate_kind == UMEM_GATE_CHANNEL;
  // the widest rows have only y in flight ahead; h and the gate come while y is summed
  constexpr bool kAhead = !kWide<G, PER>;
  size_t at = static_cast<size_t>(row) * d;
  RawRow<YT, PER> y_ahead = load_raw<G, PER, END>(y + at, lane, d), g_ahead{};
  RawRow<HT, PER> h_ahead{};
  if constexpr (kAhead) {
    h_ahead = load_raw<G, PER, END>(h + at, lane, d);
    if (gated) g_ahead = load_raw<G, PER, END>(full + at, lane, d);
  }
  const Params<G, PER, END> gamma(k.gamma, 1.f, lane, d), beta(k.beta, 0.f, lane, d);
  const Params<G, PER, END> gamma2(k.gamma_next, 1.f, lane, d), beta2(k.beta_next, 0.f, lane, d);
  Params<G, PER, END> channel(by_channel ? static_cast<const float*>(k.gate) : nullptr, 1.f, lane, d);
  if (channel.kKept && by_channel && k.sigmoid) sigmoid_row(channel.kept);
  for (; row < k.T; row += k.stride) {
    at = static_cast<size_t>(row) * d;
    Row<PER> m = widen<G, END>(y_ahead, lane, d);
    if constexpr (!kAhead) {
      h_ahead = load_raw<G, PER, END>(h + at, lane, d);
      if (gated) g_ahead = load_raw<G, PER, END>(full + at, lane, d);
    }
    const RawRow<HT, PER> h_now = h_ahead;
    const RawRow<YT, PER> g_now = g_ahead;
    if (row + k.stride < k.T) {
      const size_t next = static_cast<size_t>(row + k.stride) * d;
      y_ahead = load_raw<G, PER, END>(y + next, lane, d);
      if constexpr (kAhead) {
        h_ahead = load_raw<G, PER, END>(h + next, lane, d);
        if (gated) g_ahead = load_raw<G, PER, END>(full + next, lane, d);
      }
    }
    float token = k.s;
    if (k.gate_kind == UMEM_GATE_TOKEN) {
      const float z = static_cast<const float*>(k.gate)[row];
      token *= k.sigmoid ? sigmoid(z) : z;
    }
    if (norm) {
      normalise<G, END>(m, lane, d, k.norm_out == UMEM_NORM_LAYER, k.eps, gs);
      m = affine(m, gamma.row(lane, d), beta.row(lane, d));
    }
    Row<PER> r = widen<G, END>(h_now, lane, d), g = gated ? widen<G, END>(g_now, lane, d) : channel.row(lane, d);
    if (k.sigmoid && (gated || (!channel.kKept && by_channel))) sigmoid_row(g);
    // the next entry's norm is taken of the stream as it is stored
#pragma unroll
    for (int p = 0; p < PER; ++p)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float v = fmaf(k.a, r.v[p][i], token * (g.v[p][i] * m.v[p][i]));
        r.v[p][i] = in_row<G, END>(p, i, lane, d) ? static_cast<float>(static_cast<HT>(v)) : 0.f;
      }
    store_row<G, END>(static_cast<HT*>(k.h_out) + at, r, lane, d);
    if (k.n_next == nullptr) continue;
    normalise<G, END>(r, lane, d, k.centre_next, k.eps, gs);
    store_row<G, END>(static_cast<YT*>(k.n_next) + at, affine(r, gamma2.row(lane, d), beta2.row(lane, d)), lane, d);
  }
}

// Rows of 4,097 to 8,192 (row_shape): 1,024 threads a row.  With 512 the exit spills registers (2,048 fp32 rows of
// 8,192 105 us, 80 so), and the entry, which has to add in the exit's order to give its n', gains little (bf16
// 14.1 us, 16.5 so).
constexpr int kFours8K = 2;
constexpr int kMaxWorkgroups = 2048;         // eight of 256 threads on each of 256 CUs

}  // namespace

hipError_t launch_block_in(const umem_block_desc& bd, int T, const void* h, const float* gamma, const float* beta,
                           void* n, hipStream_t s) {
  clear_stale_error();
  const RowShape shape = row_shape(bd.d, kFours8K);
  const int wgs = row_workgroups(shape, T, kMaxWorkgroups);
  const EntryArgs k{h, gamma, beta, n, T, bd.d, wgs * (shape.group == 64 ? 4 : 1), bd.norm_in == UMEM_NORM_LAYER,
                    bd.eps};
#define UMEM_ROW_GO(K, THR) hipLaunchKernelGGL(K, dim3(wgs), dim3(THR), 0, s, k)
  UMEM_ROW_LAUNCH(entry_kernel, kFours8K)
  return hipGetLastError();
}

hipError_t launch_block_out(const umem_block_desc& bd, int T, const void* h, const void* y, const void* gate,
                            const float* gamma, const float* beta, void* h_out, const float* gamma_next,
                            const float* beta_next, void* n_next, hipStream_t s) {
  clear_stale_error();
  const RowShape shape = row_shape(bd.d, kFours8K);
  const int wgs = row_workgroups(shape, T, kMaxWorkgroups);
  const ExitArgs k{h, y, gate, gamma, beta, gamma_next, beta_next, h_out, n_next, T, bd.d,
                   wgs * (shape.group == 64 ? 4 : 1), bd.norm_out, bd.gate, bd.gate_act == UMEM_ACT_SIGMOID,
                   bd.norm_in == UMEM_NORM_LAYER, bd.eps, bd.res_scale, bd.out_scale};
  UMEM_ROW_LAUNCH(exit_kernel, kFours8K)
#undef UMEM_ROW_GO
  return hipGetLastError();
}

}  // namespace umem
