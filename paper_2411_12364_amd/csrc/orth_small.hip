// Newton-Schulz updates of matrices whose smaller side is at most 64.  The steps are polynomials of A_0 = X_0 X_0^T,
// which commute, so they run on m x m matrices alone:
//
//   P = a I + b A + c A^2,  Q <- Q P,  A <- P A P;   out = decay out + scale Q X_0
//
// and X is read twice and written once, instead of 15 launches that wait for each other.  Taken so, what A_0 loses grows where
// X's singular values are small, by a^2 a step, and with the halves of a tile on the diagonal a rounding apart, as they
// are here, by up to |a|^3; where A's noise is below 0 nothing ends that.  So all of it is fp64 (v_mfma_f64_16x16x4), and
// a pass takes no more steps than |a|^(3 steps) <= 2^33 allows (6 of a = 3.4445), which leaves 2^-20 of such a direction.
// More steps go in passes of near the same length, X between them in fp64 and its A formed again: rank 1 in 16 steps
// 1e-7 off in three passes, in one 10^6 times its size.  (Halves made equal would allow 9 steps a pass, at 2 percent more time.)
// Three launches a pass: pieces of G G^T and with them |G|^2 (its trace), the steps, a workgroup a matrix in LDS, and Q G.
// Bounded by the chain of 4 small products a step: 64 x 448 in 5 steps 130 us by the large matrices' products, so 45 (5 +
// 34 + 6).
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "umem_internal.h"

namespace umem {
namespace {

typedef double f64x4 __attribute__((ext_vector_type(4)));

constexpr int kThreads = 256, kStepThreads = 1024;
constexpr int kSide = kMaxOrthSmall, kPitch = kSide + 2, kTilePitch = kSide + 4;
constexpr int kMostChunks = 32;
static_assert(kSide == 64, "16 waves of a 16 x 16 tile each");

// The f64 operands' layout: lane l holds row (or column) l % 16, k = l / 16; of D row l / 16 + 4 r, column l % 16.
__device__ __forceinline__ f64x4 mfma64(double a, double b, f64x4 c) {
  return __builtin_amdgcn_mfma_f64_16x16x4f64(a, b, c, 0, 0, 0);
}

// How a value of G, or of X between passes, is held.
template <typename T>
using Held = std::conditional_t<std::is_same_v<T, double>, double, float>;

// A 64-wide slice of G's longer side into registers, and from there into LDS as [smaller side][longer side] with zeros
// past both.
template <typename T, bool TALL, int THREADS = kThreads>
struct Slice {
  static constexpr int kEach = kSide * 64 / THREADS;
  Held<T> v[kEach];
  __device__ __forceinline__ void load(const T* g, int m, int64_t k, int64_t k0) {
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      const int in = threadIdx.x % 64, out = threadIdx.x / 64 + THREADS / 64 * i;       // in: along G's rows
      const int s = TALL ? in : out;
      const int64_t l = k0 + (TALL ? out : in);
      v[i] = s < m && l < k ? static_cast<Held<T>>(g[TALL ? l * m + s : s * k + l]) : Held<T>(0);
    }
  }
  __device__ __forceinline__ void store(Held<T> (*t)[kTilePitch]) const {
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      const int in = threadIdx.x % 64, out = threadIdx.x / 64 + THREADS / 64 * i;
      t[TALL ? in : out][TALL ? out : in] = v[i];
    }
  }
};

// A piece of G G^T (of G^T G where G is tall) over a chunk of the longer side, to pieces[matrix][chunk][64][64].
template <typename T, bool TALL>
__global__ __launch_bounds__(kThreads) void orth_small_gram_kernel(const T* __restrict__ g, int m, int k, int chunks,
                                                                   double* __restrict__ pieces) {
  __shared__ Held<T> t[kSide][kTilePitch];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int i0 = (wave >> 1) * 32, j0 = (wave & 1) * 32;
  const int64_t mat = blockIdx.y;
  const T* x = g + mat * m * static_cast<int64_t>(k);
  const int slices = (k + 63) / 64;
  const int from = static_cast<int>(static_cast<int64_t>(slices) * blockIdx.x / chunks);
  const int to = static_cast<int>(static_cast<int64_t>(slices) * (blockIdx.x + 1) / chunks);
  const bool on = i0 < m && j0 < m;
  f64x4 acc[2][2];
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j) acc[i][j] = f64x4{0.0, 0.0, 0.0, 0.0};
  Slice<T, TALL> s;
  s.load(x, m, k, static_cast<int64_t>(from) * 64);
  for (int c = from; c < to; ++c) {
    __syncthreads();
    s.store(t);
    __syncthreads();
    if (c + 1 < to) s.load(x, m, k, static_cast<int64_t>(c + 1) * 64);
    if (!on) continue;
#pragma unroll 4
    for (int q0 = 0; q0 < 64; q0 += 4) {
      const int q = q0 + (lane >> 4);
      double a[2], b[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        a[i] = t[i0 + i * 16 + (lane & 15)][q];
        b[i] = t[j0 + i * 16 + (lane & 15)][q];
      }
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j) acc[i][j] = mfma64(a[i], b[j], acc[i][j]);
    }
  }
  double* out = pieces + (mat * chunks + blockIdx.x) * kSide * kSide;
  if (!on) return;
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int r = 0; r < 4; ++r)
        out[(i0 + i * 16 + (lane >> 4) + 4 * r) * kSide + j0 + j * 16 + (lane & 15)] = acc[i][j][r];
}

// The steps of one matrix of at most TOP rows: q[matrix][64][64] = Q / (|G| + eps), in a pass after the first Q alone.  The
// matrices are symmetric: the 16 x 16 tiles on and below the diagonal are made, a wave's at a time, and written to both
// places.  T and the next Q, which read the same, are made together: 20 tiles on 16 waves.  What bounds it is the fp64
// rate of one CU: 64^3 products of a full square are 4,096 clocks, and 5 steps have 17 squares (with full squares 42 us,
// so 34).
template <int TOP>
__global__ __launch_bounds__(kStepThreads) void orth_small_steps_kernel(const double* __restrict__ pieces, int m, int chunks,
                                                                        int steps, bool first, double a, double b,
                                                                        double c, float eps, double* __restrict__ q) {
  constexpr int kSquare = TOP / 16, kTiles = kSquare * (kSquare + 1) / 2, kWaves = kStepThreads / 64;
  static_assert(kTiles <= kWaves && 2 * kTiles <= kTiles + kWaves, "a wave has one tile of Q at most");
  __shared__ double A[kSide][kPitch], P[kSide][kPitch], Q[kSide][kPitch], T[kSide][kPitch];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t mat = blockIdx.x;
  const double* from = pieces + mat * chunks * kSide * kSide;
  constexpr int kEach = (TOP * TOP + kStepThreads - 1) / kStepThreads;
  double v[kEach] = {};
#pragma unroll 4
  for (int p = 0; p < chunks; ++p)
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      const int at = min(i * kStepThreads + static_cast<int>(threadIdx.x), TOP * TOP - 1);
      v[i] += from[(static_cast<int64_t>(p) * kSide + at / TOP) * kSide + at % TOP];
    }
#pragma unroll
  for (int i = 0; i < kEach; ++i) {
    const int at = i * kStepThreads + threadIdx.x;
    if (at < TOP * TOP) A[at / TOP][at % TOP] = v[i];
  }
  __syncthreads();
  double trace = lane < m ? A[lane][lane] : 0.0;
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) trace += __shfl_xor(trace, off, 64);
  const double norm = sqrt(trace) + static_cast<double>(eps), inverse = first ? 1.0 / norm : 1.0;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kEach; ++i) {
    const int at = i * kStepThreads + threadIdx.x, row = at / TOP, col = at % TOP;
    if (at < TOP * TOP) A[row][col] = row < m && col < m ? v[i] * inverse * inverse : 0.0;
  }
  __syncthreads();
  const auto row_of = [](int tile) { return (tile >= 1) + (tile >= 3) + (tile >= 6); };
  const auto col_of = [&](int tile) { return tile - row_of(tile) * (row_of(tile) + 1) / 2; };
  const auto times = [&](double (*x)[kPitch], double (*y)[kPitch], int tile) {
    const int i0 = row_of(tile) * 16 + (lane & 15), j0 = col_of(tile) * 16 + (lane & 15);
    f64x4 acc = {0.0, 0.0, 0.0, 0.0};
#pragma unroll
    for (int k0 = 0; k0 < TOP; k0 += 4) {
      const int k = k0 + (lane >> 4);
      acc = mfma64(x[i0][k], y[j0][k], acc);
    }
    return acc;
  };
  const auto put = [&](double (*x)[kPitch], const f64x4& v, int tile) {
    const int i0 = row_of(tile) * 16 + (lane >> 4), j = col_of(tile) * 16 + (lane & 15);
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      x[i0 + 4 * r][j] = v[r];
      x[j][i0 + 4 * r] = v[r];            // (a tile on the diagonal: the other half of it, equal but for a rounding)
    }
  };
  for (int step = 0; step < steps; ++step) {
    if (wave < kTiles) {
      f64x4 p = times(A, A, wave);
      const int i0 = row_of(wave) * 16 + (lane >> 4), j = col_of(wave) * 16 + (lane & 15);
#pragma unroll
      for (int r = 0; r < 4; ++r) p[r] = c * p[r] + b * A[i0 + 4 * r][j] + (i0 + 4 * r == j ? a : 0.0);
      put(P, p, wave);
      if (step == 0) put(Q, p, wave);
    }
    __syncthreads();
    const bool last = step + 1 == steps;
    const int of_t = last ? 0 : kTiles, of_q = step == 0 ? 0 : kTiles;
    f64x4 next = {0.0, 0.0, 0.0, 0.0};
    int mine = -1;                        // the wave's tile of the next Q, which takes the place of the one that is read
    for (int task = wave; task < of_t + of_q; task += kWaves) {
      if (task < of_t) {
        put(T, times(P, A, task), task);
      } else {
        mine = task - of_t;
        next = times(Q, P, mine);
      }
    }
    __syncthreads();
    if (mine >= 0) put(Q, next, mine);
    if (last) break;
    if (wave < kTiles) put(A, times(P, T, wave), wave);
    __syncthreads();
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kEach; ++i) {
    const int at = i * kStepThreads + threadIdx.x, row = at / TOP, col = at % TOP;
    if (at < TOP * TOP) q[(mat * kSide + row) * kSide + col] = Q[row][col] * inverse;
  }
}

// out = decay out + scale Q G (G Q where G is tall) over 64 of the longer side, a 16 x 16 block a wave (with four blocks a
// wave, one wave to each of a CU's parts, 64 x 448 took 10 us, so 5.6).
template <typename GT, typename OT, bool TALL>
__global__ __launch_bounds__(kStepThreads) void orth_small_apply_kernel(const GT* g, int m, int k, const double* __restrict__ q,
                                                                        OT* out, float decay, float scale) {
  __shared__ double Q[kSide][kPitch];
  __shared__ Held<GT> t[kSide][kTilePitch];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, i0 = (wave >> 2) * 16, l0 = (wave & 3) * 16;
  const int64_t mat = blockIdx.y, k0 = static_cast<int64_t>(blockIdx.x) * 64, base = mat * m * static_cast<int64_t>(k);
  Slice<GT, TALL, kStepThreads> s;
  s.load(g + base, m, k, k0);
#pragma unroll
  for (int i = 0; i < kSide * kSide / kStepThreads; ++i) {
    const int at = i * kStepThreads + threadIdx.x, row = at / kSide, col = at % kSide;
    Q[row][col] = row < m && col < m ? q[mat * kSide * kSide + at] : 0.0;
  }
  s.store(t);
  __syncthreads();
  if (i0 >= m) return;
  f64x4 acc = {0.0, 0.0, 0.0, 0.0};
#pragma unroll
  for (int j0 = 0; j0 < kSide; j0 += 4) {
    const int j = j0 + (lane >> 4);
    const double x = t[j][l0 + (lane & 15)], w = Q[i0 + (lane & 15)][j];
    acc = TALL ? mfma64(x, w, acc) : mfma64(w, x, acc);
  }
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    const int a = (lane >> 4) + 4 * r, b = lane & 15;
    const int small = i0 + (TALL ? b : a);
    const int64_t at = k0 + l0 + (TALL ? a : b);
    if (small >= m || at >= k) continue;
    OT* to = out + base + (TALL ? at * m + small : small * static_cast<int64_t>(k) + at);
    double v = static_cast<double>(scale) * acc[r];
    if constexpr (std::is_same_v<OT, double>) {             // (X between passes)
      *to = v;
    } else {
      if (decay != 0.f) v = fma(static_cast<double>(decay), static_cast<double>(static_cast<float>(*to)), v);
      *to = static_cast<OT>(static_cast<float>(v));
    }
  }
}

size_t up256(size_t x) { return (x + 255) & ~static_cast<size_t>(255); }

// Chunks of the longer side: few enough that adding their pieces costs little, and 1,024 workgroups at most.
int chunk_count(const umem_orth_desc& od) {
  const int slices = (std::max(od.rows, od.cols) + 63) / 64;
  return std::min(slices, std::min(kMostChunks, std::max(1, 1024 / od.n)));
}

// How the steps are taken: in passes of at most as many as the growth of what A loses allows, the longer ones first.
struct Passes {
  int count;
  explicit Passes(const umem_orth_desc& od) {
    int most = od.steps;
    while (most > 1 && std::pow(std::fabs(static_cast<double>(od.a)), 3 * most) > 0x1p33) --most;
    count = (od.steps + most - 1) / most;
  }
  int of(int pass, int steps) const { return steps / count + (pass < steps % count ? 1 : 0); }
};

// X between the passes lies where the workspace's other parts end; it is read and written by the same workgroups.
struct SmallLayout {
  size_t q, x, total;
  explicit SmallLayout(const umem_orth_desc& od) {
    const size_t n = od.n, square = kSide * kSide * sizeof(double);
    q = up256(n * chunk_count(od) * square);
    x = q + up256(n * square);
    total = x + (Passes(od).count > 1 ? up256(n * od.rows * od.cols * sizeof(double)) : 0);
  }
};

struct SmallRun {
  const umem_orth_desc& od;
  double *pieces, *q;
  hipStream_t s;

  template <bool TALL, typename GT, typename OT>
  void pass(const GT* g, OT* out, int steps, bool first, float decay, float scale) const {
    const int m = std::min(od.rows, od.cols), k = std::max(od.rows, od.cols), chunks = chunk_count(od);
    hipLaunchKernelGGL((orth_small_gram_kernel<GT, TALL>), dim3(chunks, od.n), dim3(kThreads), 0, s, g, m, k, chunks, pieces);
    const auto step = m <= 16   ? orth_small_steps_kernel<16>
                      : m <= 32 ? orth_small_steps_kernel<32>
                      : m <= 48 ? orth_small_steps_kernel<48>
                                : orth_small_steps_kernel<64>;
    hipLaunchKernelGGL(step, dim3(od.n), dim3(kStepThreads), 0, s, pieces, m, chunks, steps, first,
                       static_cast<double>(od.a), static_cast<double>(od.b), static_cast<double>(od.c), od.eps, q);
    hipLaunchKernelGGL((orth_small_apply_kernel<GT, OT, TALL>), dim3((k + 63) / 64, od.n), dim3(kStepThreads), 0, s, g, m, k,
                       q, out, decay, scale);
  }

  template <bool TALL, typename GT, typename OT>
  void all(const GT* g, OT* out, double* x) const {
    const Passes p(od);
    if (p.count == 1) {
      pass<TALL>(g, out, od.steps, true, od.decay, od.scale);
      return;
    }
    for (int i = 0; i < p.count; ++i) {
      const int steps = p.of(i, od.steps);
      if (i == 0) pass<TALL>(g, x, steps, true, 0.f, 1.f);
      else if (i + 1 < p.count) pass<TALL>(static_cast<const double*>(x), x, steps, false, 0.f, 1.f);
      else pass<TALL>(static_cast<const double*>(x), out, steps, false, od.decay, od.scale);
    }
  }
};

}  // namespace

size_t orth_small_workspace_bytes(const umem_orth_desc& od) { return SmallLayout(od).total; }

hipError_t launch_orth_small(const umem_orth_desc& od, const void* g, void* out, void* ws, hipStream_t s) {
  clear_stale_error();
  const SmallLayout L(od);
  char* base = static_cast<char*>(ws);
  const SmallRun run{od, reinterpret_cast<double*>(base), reinterpret_cast<double*>(base + L.q), s};
  double* between = reinterpret_cast<double*>(base + L.x);
  const auto go = [&](auto* x, auto* y) {
    if (od.rows > od.cols) run.all<true>(x, y, between);
    else run.all<false>(x, y, between);
  };
  const auto from = [&](auto* x) {
    if (od.otype == UMEM_F32) go(x, static_cast<float*>(out));
    else go(x, static_cast<__bf16*>(out));
  };
  if (od.gtype == UMEM_F32) from(static_cast<const float*>(g));
  else from(static_cast<const __bf16*>(g));
  return hipGetLastError();
}

}  // namespace umem
