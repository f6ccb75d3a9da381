// The backward of the norms before and after a block (block.hip).
//
// With v = gamma * (gradient of Norm's output) and r = 1 / spread, per row
//   dx = r (v - mean(v) - x^ mean(v x^))          (mean(v) for LayerNorm only)
// and over the rows  dgamma = sum dn x^,  dbeta = sum dn,  a channel gate's gradient.
//
// The statistics are recomputed from the row, which has to be read in any case: mean(v) is summed beside the
// row's mean, and v's product with the centred row beside its variance, so a row takes two rounds of sums
// over its group (RMS: one).  A group walks rows with its columns' parameters and column sums in registers,
// the next row's loads in flight; the workgroups' column sums are added up in order by a second kernel.
#include "block_rows.h"

namespace umem {
namespace {

struct EntryBackArgs {
  const void *h, *dn, *dres;
  const float* gamma;
  void* dh;
  float* part;                 // [workgroups][dgamma, dbeta][d]
  int T, d, stride;
  bool centre, shift;
  float eps;
};

struct ExitBackArgs {
  const void *y, *gate, *dh_out;
  const float *gamma, *beta;
  void *dh, *dy, *dgate;
  float* part;                 // [workgroups][dgamma, dbeta, dgate of a channel gate][d], those there are
  int T, d, stride, norm_out, gate_kind;
  bool sigmoid;
  float eps, a, s;
};

// A group's column sums: in registers, or, of the widest rows, whose threads have none left, each thread's own
// in LDS (no thread reads another's, so nothing waits): 1,024 fp32 rows of 12,288 leave the exit's backward in
// 112 us, with the sums in registers, of which more are spilled then, 172, the entry's in 46 and 67.
template <int G, int PER>
struct ColumnSums {
  static constexpr bool kLds = kWide<G, PER>;
  Row<PER> kept;
  rf32x4* mine;
  __device__ __forceinline__ ColumnSums(float* lds, int which) : kept{} {
    if constexpr (kLds) {
      mine = reinterpret_cast<rf32x4*>(lds) + which * PER * G + threadIdx.x;
#pragma unroll
      for (int p = 0; p < PER; ++p) mine[p * G] = 0.f;
    }
  }
  __device__ __forceinline__ rf32x4 at(int p) const {
    if constexpr (kLds) return mine[p * G];
    else return kept.v[p];
  }
  __device__ __forceinline__ void put(int p, rf32x4 v) {
    if constexpr (kLds) mine[p * G] = v;
    else kept.v[p] = v;
  }
  __device__ __forceinline__ Row<PER> all() const {
    Row<PER> r;
#pragma unroll
    for (int p = 0; p < PER; ++p) r.v[p] = at(p);
    return r;
  }
};
// Bytes of two of them.
inline size_t column_lds(const RowShape& s) { return s.group == 1024 && s.per == 4 ? 2u * 4 * 1024 * 16 : 0; }

// x -> x^, and r with the two means of the backward.
struct BackSums {
  float r, s0, s1;
};
template <int G, RowEnd END, int PER>
__device__ __forceinline__ BackSums back_sums(Row<PER>& x, const Row<PER>& v, int lane, int d, bool centre, float eps,
                                              GroupSum<G>& gs) {
  const float inv_d = 1.0f / static_cast<float>(d);
  BackSums b{0.f, 0.f, 0.f};
  if (centre) {
    float sx = add_up(x), sv = add_up(v);
    gs.sum2(sx, sv);
    b.s0 = sv * inv_d;
    centre_row<G, END>(x, sx * inv_d, lane, d);
  }
  float q = dot(x, x), vx = dot(v, x);
  gs.sum2(q, vx);
  b.r = rsqrtf(q * inv_d + eps);
  b.s1 = vx * b.r * inv_d;
#pragma unroll
  for (int p = 0; p < PER; ++p) x.v[p] *= b.r;
  return b;
}

// A workgroup's column sums to its place of the partial sums: its groups' are added in order in LDS.
template <int G, RowEnd END, int PER>
__device__ __forceinline__ void write_part(const Row<PER>& acc, float* part, int lane, int d, float* lds) {
  Row<PER> s = acc;
  if constexpr (Group<G>::kRows > 1) {
#pragma unroll
    for (int p = 0; p < PER; ++p) {
      __syncthreads();
      *reinterpret_cast<rf32x4*>(lds + threadIdx.x * 4) = acc.v[p];
      __syncthreads();
#pragma unroll
      for (int w = 1; w < Group<G>::kRows; ++w) s.v[p] += *reinterpret_cast<const rf32x4*>(lds + (w * G + lane) * 4);
    }
    if (Group<G>::index() != 0) return;      // (its s starts from its own sums)
  }
  store_row<G, END>(part, s, lane, d);
}

template <typename HT, typename YT, int G, int PER, RowEnd END>
__global__ __launch_bounds__(Group<G>::kThreads) void entry_back_kernel(EntryBackArgs k) {
  __shared__ float lds[2][Group<G>::kWaves][2];
  __shared__ __align__(16) float sums[Group<G>::kRows > 1 ? 1024 : 4];
  const int lane = Group<G>::lane(), d = k.d;
  GroupSum<G> gs{lds, 0};
  const HT *h = static_cast<const HT*>(k.h), *dres = static_cast<const HT*>(k.dres);
  const YT* dn = static_cast<const YT*>(k.dn);
  const bool more = dres != nullptr;
  extern __shared__ __align__(16) float wide[];
  ColumnSums<G, PER> dg(wide, 0), db(wide, 1);
  int row = blockIdx.x * Group<G>::kRows + Group<G>::index();
  RawRow<HT, PER> h_ahead{}, u_ahead{};
  RawRow<YT, PER> n_ahead{};
  auto load = [&](int r) {
    const size_t at = static_cast<size_t>(r) * d;
    h_ahead = load_raw<G, PER, END>(h + at, lane, d);
    n_ahead = load_raw<G, PER, END>(dn + at, lane, d);
    if (more) u_ahead = load_raw<G, PER, END>(dres + at, lane, d);
  };
  constexpr bool kAhead = !kWide<G, PER>;
  if (kAhead && row < k.T) load(row);
  const Params<G, PER, END> of_gamma(k.gamma, 1.f, lane, d);
  for (; row < k.T; row += k.stride) {
    if (!kAhead) load(row);
    const Row<PER> n = widen<G, END>(n_ahead, lane, d), up = widen<G, END>(u_ahead, lane, d),
                   gamma = of_gamma.row(lane, d);
    Row<PER> x = widen<G, END>(h_ahead, lane, d), v;
    if (kAhead && row + k.stride < k.T) load(row + k.stride);
#pragma unroll
    for (int p = 0; p < PER; ++p) v.v[p] = n.v[p] * gamma.v[p];
    const BackSums b = back_sums<G, END>(x, v, lane, d, k.centre, k.eps, gs);
#pragma unroll
    for (int p = 0; p < PER; ++p) {
      rf32x4 sg = dg.at(p);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float xh = x.v[p][i];
        sg[i] = fmaf(n.v[p][i], xh, sg[i]);
        v.v[p][i] = fmaf(v.v[p][i] - b.s0 - xh * b.s1, b.r, up.v[p][i]);
      }
      dg.put(p, sg);
      db.put(p, db.at(p) + n.v[p]);
    }
    store_row<G, END>(static_cast<HT*>(k.dh) + static_cast<size_t>(row) * d, v, lane, d);
  }
  float* part = k.part + static_cast<size_t>(blockIdx.x) * (k.shift ? 2 : 1) * d;
  write_part<G, END>(dg.all(), part, lane, d, sums);
  if (k.shift) write_part<G, END>(db.all(), part + d, lane, d, sums);
}

template <typename HT, typename YT, int G, int PER, RowEnd END>
__global__ __launch_bounds__(Group<G>::kThreads) void exit_back_kernel(ExitBackArgs k) {
  __shared__ float lds[2][Group<G>::kWaves][2];
  __shared__ __align__(16) float sums[Group<G>::kRows > 1 ? 1024 : 4];
  const int lane = Group<G>::lane(), d = k.d;
  const bool norm = k.norm_out != UMEM_NORM_NONE, full = k.gate_kind == UMEM_GATE_FULL,
             channel = k.gate_kind == UMEM_GATE_CHANNEL, token = k.gate_kind == UMEM_GATE_TOKEN;
  GroupSum<G> gs{lds, 0};
  const HT* dh_out = static_cast<const HT*>(k.dh_out);
  const YT *y = static_cast<const YT*>(k.y), *gate = static_cast<const YT*>(k.gate);
  extern __shared__ __align__(16) float wide[];
  ColumnSums<G, PER> dg(wide, 0), db(wide, 1);
  Row<PER> dc{};
  int row = blockIdx.x * Group<G>::kRows + Group<G>::index();
  RawRow<YT, PER> y_ahead{}, g_ahead{};
  RawRow<HT, PER> h_ahead{};
  auto load = [&](int r) {
    const size_t at = static_cast<size_t>(r) * d;
    y_ahead = load_raw<G, PER, END>(y + at, lane, d);
    h_ahead = load_raw<G, PER, END>(dh_out + at, lane, d);
    if (full) g_ahead = load_raw<G, PER, END>(gate + at, lane, d);
  };
  constexpr bool kAhead = !kWide<G, PER>;
  if (kAhead && row < k.T) load(row);
  const Params<G, PER, END> of_gamma(k.gamma, 1.f, lane, d), of_beta(k.beta, 0.f, lane, d);
  // a channel gate's value; its slope comes from it
  Params<G, PER, END> value(channel ? static_cast<const float*>(k.gate) : nullptr, 1.f, lane, d);
  if (value.kKept && channel && k.sigmoid) sigmoid_row(value.kept);
  for (; row < k.T; row += k.stride) {
    const size_t at = static_cast<size_t>(row) * d;
    if (!kAhead) load(row);
    Row<PER> x = widen<G, END>(y_ahead, lane, d), up = widen<G, END>(h_ahead, lane, d), v;
    Row<PER> g = full ? widen<G, END>(g_ahead, lane, d) : value.row(lane, d);
    if (kAhead && row + k.stride < k.T) load(row + k.stride);
    if (k.dh != nullptr) {
#pragma unroll
      for (int p = 0; p < PER; ++p) v.v[p] = up.v[p] * k.a;
      store_row<G, END>(static_cast<HT*>(k.dh) + at, v, lane, d);
    }
    if (k.sigmoid && (full || (!value.kKept && channel))) sigmoid_row(g);
    float of_token = 1.f;
    if (token) {
      of_token = static_cast<const float*>(k.gate)[row];
      if (k.sigmoid) of_token = sigmoid(of_token);
    }
    // up: out_scale dh_out, the gradient of the gated output; g: that of Norm_out's output
    Row<PER> gamma = of_gamma.row(lane, d);
#pragma unroll
    for (int p = 0; p < PER; ++p) {
      up.v[p] *= k.s;
      v.v[p] = up.v[p] * (g.v[p] * of_token) * gamma.v[p];
    }
    BackSums b{1.f, 0.f, 0.f};
    if (norm) b = back_sums<G, END>(x, v, lane, d, k.norm_out == UMEM_NORM_LAYER, k.eps, gs);
    if (!of_gamma.kKept) gamma = of_gamma.row(lane, d);
    const Row<PER> beta = of_beta.row(lane, d);
    float st = 0.f;
#pragma unroll
    for (int p = 0; p < PER; ++p) {
      rf32x4 sg = dg.at(p), sb = db.at(p);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float xh = x.v[p][i], gv = g.v[p][i];
        // the gradient of the gate's value, and of its argument
        float dz = up.v[p][i] * fmaf(xh, gamma.v[p][i], beta.v[p][i]);
        st += dz;
        if (k.sigmoid) dz *= gv * (1.0f - gv);
        const float dm = up.v[p][i] * (gv * of_token);
        sg[i] = fmaf(dm, xh, sg[i]);
        sb[i] += dm;
        dc.v[p][i] += dz;
        up.v[p][i] = dz;
        v.v[p][i] = norm ? (v.v[p][i] - b.s0 - xh * b.s1) * b.r : v.v[p][i];
      }
      dg.put(p, sg);
      db.put(p, sb);
    }
    if (full) store_row<G, END>(static_cast<YT*>(k.dgate) + at, up, lane, d);
    store_row<G, END>(static_cast<YT*>(k.dy) + at, v, lane, d);
    if (token) {
      st = gs.sum(st);
      if (lane == 0) static_cast<float*>(k.dgate)[row] = k.sigmoid ? st * (of_token * (1.0f - of_token)) : st;
    }
  }
  const int q = (norm ? 1 : 0) + (k.beta != nullptr ? 1 : 0) + (channel ? 1 : 0);
  float* part = k.part + static_cast<size_t>(blockIdx.x) * q * d;
  if (norm) {
    write_part<G, END>(dg.all(), part, lane, d, sums);
    part += d;
  }
  if (k.beta != nullptr) {
    write_part<G, END>(db.all(), part, lane, d, sums);
    part += d;
  }
  if (channel) write_part<G, END>(dc, part, lane, d, sums);
}

// The column sums: 128 threads take every 128th partial row each, in order, of four columns, and theirs
// are added in a fixed tree, so that the result does not depend on timing.
struct ColumnArgs {
  const float* part;
  float* out[3];
  int q, d, parts;
  bool accumulate;
};

constexpr int kColWide = 8, kColDeep = 128;  // threads: 32 columns, 128 bytes of a partial row
__global__ __launch_bounds__(kColWide * kColDeep) void column_sum_kernel(ColumnArgs k) {
  __shared__ rf32x4 lds[kColDeep][kColWide];
  const int x = threadIdx.x % kColWide, deep = threadIdx.x / kColWide;
  const int n = k.q * k.d, c = (blockIdx.x * kColWide + x) * 4;
  rf32x4 s = {0.f, 0.f, 0.f, 0.f};
  if (c + 4 <= n) {
#pragma unroll 4
    for (int w = deep; w < k.parts; w += kColDeep)
      s += *reinterpret_cast<const Quad<float>::type*>(k.part + static_cast<size_t>(w) * n + c);
  } else if (c < n) {
    for (int w = deep; w < k.parts; w += kColDeep)
      for (int i = 0; i < n - c; ++i) s[i] += k.part[static_cast<size_t>(w) * n + c + i];
  }
  lds[deep][x] = s;
#pragma unroll
  for (int half = kColDeep / 2; half > 0; half >>= 1) {
    __syncthreads();
    if (deep < half) lds[deep][x] += lds[deep + half][x];
  }
  if (deep != 0) return;
  s = lds[0][x];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (c + i >= n) break;
    const int which = (c + i) / k.d;
    float* out = (which == 0 ? k.out[0] : which == 1 ? k.out[1] : k.out[2]) + (c + i - which * k.d);
    *out = k.accumulate ? *out + s[i] : s[i];
  }
}

// Workgroups of a backward, and its rows of partial sums: two for each CU, or one of 512 threads or more, whose
// rows are as many bytes (exit's backward of 2,048 bf16 rows of 4,096 31.5 us, with two 34, of 300 rows 13 and
// 16; 8,192 bf16 rows of 2,048 take 49 with two workgroups of 256 threads, 59 with one).
int most_parts(const RowShape& s) { return s.group >= 512 ? 256 : 512; }
// Rows of 4,097 to 8,192 (row_shape), 512 threads a row: the exit's backward of 2,048 fp32 rows of 5,000 79 us, with 1,024
// threads 112; bf16 43 and 62.  Both spill: 2 to 98 registers in nine of twelve instances, with 1,024
// threads 23 to 112 in all.
constexpr int kFours8K = 4;

hipError_t launch_columns(const ColumnArgs& c, hipStream_t s) {
  const int n = c.q * c.d;
  hipLaunchKernelGGL(column_sum_kernel, dim3((n + 4 * kColWide - 1) / (4 * kColWide)), dim3(kColWide * kColDeep), 0, s, c);
  return hipGetLastError();
}

}  // namespace

// A workgroup's row of partial sums for each of the most workgroups that T rows or fewer take: row_workgroups
// itself falls where another turn of rows begins (512 rows of 2,048: 512 workgroups; 513: 257), and a
// workspace sized once for the longest batch has to do for the shorter ones.
size_t block_backward_workspace_bytes(const umem_block_desc& bd, int T) {
  if (T == 0) return 0;
  const RowShape shape = row_shape(bd.d, kFours8K);
  const size_t bytes = static_cast<size_t>(std::min(row_groups(shape, T), most_parts(shape))) * 3 * bd.d * sizeof(float);
  return (bytes + 255) / 256 * 256;
}

hipError_t launch_block_in_backward(const umem_block_desc& bd, int T, const void* h, const float* gamma,
                                    const void* dn, const void* dres, void* dh, float* dgamma, float* dbeta,
                                    bool accumulate, void* ws, hipStream_t s) {
  clear_stale_error();
  const RowShape shape = row_shape(bd.d, kFours8K);
  const int wgs = row_workgroups(shape, T, most_parts(shape));
  const EntryBackArgs k{h, dn, dres, gamma, dh, static_cast<float*>(ws), T, bd.d, wgs * (shape.group == 64 ? 4 : 1),
                        bd.norm_in == UMEM_NORM_LAYER, dbeta != nullptr, bd.eps};
#define UMEM_ROW_GO(K, THR) hipLaunchKernelGGL(K, dim3(wgs), dim3(THR), column_lds(shape), s, k)
  UMEM_ROW_LAUNCH(entry_back_kernel, kFours8K)
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  return launch_columns({static_cast<const float*>(ws), {dgamma, dbeta, nullptr}, dbeta ? 2 : 1, bd.d, wgs, accumulate}, s);
}

hipError_t launch_block_out_backward(const umem_block_desc& bd, int T, const void* y, const void* gate,
                                     const float* gamma, const float* beta, const void* dh_out, void* dh, void* dy,
                                     void* dgate, float* dgamma, float* dbeta, bool accumulate, void* ws,
                                     hipStream_t s) {
  clear_stale_error();
  const RowShape shape = row_shape(bd.d, kFours8K);
  const int wgs = row_workgroups(shape, T, most_parts(shape));
  const ExitBackArgs k{y, gate, dh_out, gamma, beta, dh, dy, dgate, static_cast<float*>(ws), T, bd.d,
                       wgs * (shape.group == 64 ? 4 : 1), bd.norm_out, bd.gate, bd.gate_act == UMEM_ACT_SIGMOID,
                       bd.eps, bd.res_scale, bd.out_scale};
  UMEM_ROW_LAUNCH(exit_back_kernel, kFours8K)
#undef UMEM_ROW_GO
  const hipError_t e = hipGetLastError();
  ColumnArgs c{static_cast<const float*>(ws), {nullptr, nullptr, nullptr}, 0, bd.d, wgs, accumulate};
  if (dgamma != nullptr) c.out[c.q++] = dgamma;
  if (dbeta != nullptr) c.out[c.q++] = dbeta;
  if (bd.gate == UMEM_GATE_CHANNEL) c.out[c.q++] = static_cast<float*>(dgate);
  return e != hipSuccess || c.q == 0 ? e : launch_columns(c, s);
}

}  // namespace umem
