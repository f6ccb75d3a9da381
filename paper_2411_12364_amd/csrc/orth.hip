// The orthogonalised update of a matrix by Newton-Schulz products:
//
//   X_0 = G / (|G|_F + eps),  X <- a X + (b A + c A^2) X with A = X X^T,  out = decay out + scale X_steps
//
// on the smaller side: a tall G is worked on transposed, so A is m x m with m = min(rows, cols).  All three products of a
// step have both operands with k innermost (tiles.h): A's are X's rows, A^2's are A's rows, as A is symmetric, and
// X's update takes B = b A + c A^2 and the transposed X, so X is kept in both orders.  Bounded by the matrix cores for
// large matrices, by the chain of 3 steps launches for small ones.
//
// Rounding: every matrix between the steps is two fp16 parts of its values times 2^12, which hold 22 bits of it, and
// a product takes three of the four pairs of parts (the fourth is below 2^-22 of the result); sums are fp32, |G|_F is fp64.
// Two bf16 parts would hold 17 bits: what a step loses of X's small singular values grows by a = 3.4 a step
// (a random 896 x 2,048 matrix after five steps: 4e-7 off the exact result with the fp16 parts, 2e-5 with the bf16 ones).
// An entry of X, A or B that reaches 16 becomes infinite: of coefficients that
// keep singular values of 1 near 1 none does.
#include <algorithm>

#include "tiles.h"

namespace umem {
namespace {

constexpr int kThreads = 256;
constexpr float kUp = 4096.f, kDown = 1.f / 4096.f;

__device__ __forceinline__ uint32_t f16_bits(float x) { return __builtin_bit_cast(uint16_t, static_cast<_Float16>(x)); }
__device__ __forceinline__ float bits_f32(uint32_t b) {
  return static_cast<float>(__builtin_bit_cast(_Float16, static_cast<uint16_t>(b)));
}
// x (times 2^12 already) as two parts; of one that is infinite or no number the second is zero.
__device__ __forceinline__ void f16_parts(float x, uint32_t& hi, uint32_t& lo) {
  hi = f16_bits(x);
  const float v = bits_f32(hi);
  lo = fabsf(v) < INFINITY ? f16_bits(x - v) : 0u;
}

template <typename T>
__device__ __forceinline__ float to_f32(T x) {
  return static_cast<float>(x);
}

// A matrix of [rows][ld] in two parts, one after the other, and how far the next matrix of the batch is.
struct Parts {
  uint16_t* p;
  int64_t part, ld, matrix;
};

// ---------------------------------------------------------------- norm and first X

constexpr int kNormBlocks = 64;

// |G|^2 of each matrix, in kNormBlocks fp64 pieces of fixed ranges.
template <typename T>
__global__ __launch_bounds__(kThreads) void orth_norm_kernel(const T* __restrict__ g, int64_t size,
                                                             double* __restrict__ pieces) {
  __shared__ double waves[kThreads / kWave];
  const T* m = g + blockIdx.y * size;
  double sum = 0.0;
  for (int64_t i = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x; i < size; i += kNormBlocks * kThreads) {
    const double v = to_f32(m[i]);
    sum += v * v;
  }
#pragma unroll
  for (int off = kWave / 2; off > 0; off >>= 1) sum += __shfl_xor(sum, off, kWave);
  if ((threadIdx.x & (kWave - 1)) == 0) waves[threadIdx.x / kWave] = sum;
  __syncthreads();
  if (threadIdx.x == 0) {
#pragma unroll
    for (int w = 1; w < kThreads / kWave; ++w) sum += waves[w];
    pieces[blockIdx.y * kNormBlocks + blockIdx.x] = sum;
  }
}

// X_0 in both orders, with zeros up to the rows' ends; a 64 x 64 tile of G a workgroup.  by_rows [rows][ld of cols],
// by_cols [cols][ld of rows].
template <typename T>
__global__ __launch_bounds__(kThreads) void orth_first_kernel(const T* __restrict__ g, int rows, int cols, float eps,
                                                              const double* __restrict__ pieces, Parts by_rows,
                                                              Parts by_cols) {
  __shared__ uint32_t tile[64][65];
  const int r0 = blockIdx.y * 64, c0 = blockIdx.x * 64;
  const int64_t mat = blockIdx.z;
  double sum = 0.0;
#pragma unroll 8
  for (int i = 0; i < kNormBlocks; ++i) sum += pieces[mat * kNormBlocks + i];
  const float norm = static_cast<float>(sqrt(sum)) + eps;
  const T* m = g + mat * rows * static_cast<int64_t>(cols);
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const int r = i * 4 + threadIdx.x / 64, c = threadIdx.x % 64;
    const bool in = r0 + r < rows && c0 + c < cols;
    const float v = in ? to_f32(m[(r0 + r) * static_cast<int64_t>(cols) + c0 + c]) / norm : 0.f;
    uint32_t hi, lo;
    f16_parts(v * kUp, hi, lo);
    tile[r][c] = in ? hi | lo << 16 : 0u;
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int a = i * 8 + threadIdx.x / 32, b = (threadIdx.x % 32) * 2;
    if (r0 + a < rows && c0 + b < by_rows.ld) {
      const uint32_t x = tile[a][b], y = tile[a][b + 1];
      uint16_t* to = by_rows.p + mat * by_rows.matrix + (r0 + a) * by_rows.ld + c0 + b;
      *reinterpret_cast<uint32_t*>(to) = (x & 0xffffu) | y << 16;
      *reinterpret_cast<uint32_t*>(to + by_rows.part) = x >> 16 | (y & 0xffff0000u);
    }
    if (c0 + a < cols && r0 + b < by_cols.ld) {
      const uint32_t x = tile[b][a], y = tile[b + 1][a];
      uint16_t* to = by_cols.p + mat * by_cols.matrix + (c0 + a) * by_cols.ld + r0 + b;
      *reinterpret_cast<uint32_t*>(to) = (x & 0xffffu) | y << 16;
      *reinterpret_cast<uint32_t*>(to + by_cols.part) = x >> 16 | (y & 0xffff0000u);
    }
  }
}

// ---------------------------------------------------------------- products

// Four values (times 2^12) at row n, columns m .. m + 3 of a matrix of `cols` columns, and at rows m .. m + 3, column n of
// its transpose; columns up to the pads become zeros.
__device__ __forceinline__ void put_row(const Parts& out, int64_t mat, int n, int m, int cols, f32x4 v) {
  if (m >= out.ld) return;
  uint32_t hi[4], lo[4];
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    f16_parts(v[r], hi[r], lo[r]);
    if (m + r >= cols) hi[r] = lo[r] = 0u;
  }
  uint16_t* to = out.p + mat * out.matrix + n * out.ld + m;
  *reinterpret_cast<u32x2*>(to) = u32x2{hi[0] | hi[1] << 16, hi[2] | hi[3] << 16};
  *reinterpret_cast<u32x2*>(to + out.part) = u32x2{lo[0] | lo[1] << 16, lo[2] | lo[3] << 16};
}
__device__ __forceinline__ void put_column(const Parts& out, int64_t mat, int n, int m, int rows, f32x4 v) {
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    if (m + r >= rows) break;
    uint32_t hi, lo;
    f16_parts(v[r], hi, lo);
    uint16_t* to = out.p + mat * out.matrix + (m + r) * out.ld + n;
    to[0] = static_cast<uint16_t>(hi);
    to[out.part] = static_cast<uint16_t>(lo);
  }
}
// The four values (times 2^12) at row n, columns m .. m + 3.
__device__ __forceinline__ f32x4 get_row(const Parts& in, int64_t mat, int n, int m) {
  const uint16_t* from = in.p + mat * in.matrix + n * in.ld + m;
  const u32x2 hi = *reinterpret_cast<const u32x2*>(from), lo = *reinterpret_cast<const u32x2*>(from + in.part);
  return f32x4{bits_f32(hi.x & 0xffffu) + bits_f32(lo.x & 0xffffu), bits_f32(hi.x >> 16) + bits_f32(lo.x >> 16),
               bits_f32(hi.y & 0xffffu) + bits_f32(lo.y & 0xffffu), bits_f32(hi.y >> 16) + bits_f32(lo.y >> 16)};
}

enum Mode { kGram, kPoly, kUpdate, kLast };

struct OrthArgs {
  Parts a, b;             // the product's operands: rows along m and along n, k innermost
  Parts own;              // kPoly: A; kUpdate, kLast: X by rows n, m along its rows
  Parts out, out_t;       // kGram, kPoly: the product (symmetric); kUpdate: X by rows n, and transposed
  int rows_m, rows_n, k;
  int tiles_m, tiles_n, items;
  float alpha, beta;      // kPoly: alpha A + beta A^2; kUpdate: alpha X + B X
  float decay, scale;     // kLast: final = decay final + scale (alpha X + B X), [n][m] of ld
  void* final;
  int64_t final_ld, final_matrix;
};

template <Mode MODE, typename OT, int BM, int BN, int WR, int WC>
__global__ __launch_bounds__(64 * WR * WC) void orth_product_kernel(OrthArgs g) {
  typedef Tile<true, BM, BN, WR, WC> Tl;
  __shared__ __align__(16) uint16_t buf0[Tl::kElems];
  __shared__ __align__(16) uint16_t buf1[Tl::kElems];
  const int item = tile_item(g.items);
  if (item >= g.items) return;
  constexpr bool kSym = MODE == kGram || MODE == kPoly;
  const int per = kSym ? g.tiles_m * (g.tiles_m + 1) / 2 : g.tiles_m * g.tiles_n;
  const int64_t mat = item / per;
  const int in = item - static_cast<int>(mat) * per;
  TilePlace at;
  if constexpr (kSym) {      // the lower triangle: n <= m
    int m = static_cast<int>((sqrtf(8.f * in + 1.f) - 1.f) * 0.5f);
    while ((m + 1) * (m + 2) / 2 <= in) ++m;
    while (m * (m + 1) / 2 > in) --m;
    at = {m, in - m * (m + 1) / 2};
  } else {
    at = tile_place(in, g.tiles_m, g.tiles_n);
  }
  TilePairs p;
  p.n = 3;
  const uint16_t *a = g.a.p + mat * g.a.matrix, *b = g.b.p + mat * g.b.matrix;
  p.a[0] = a;
  p.b[0] = b + g.b.part;
  p.a[1] = a + g.a.part;
  p.b[1] = b;
  p.a[2] = a;
  p.b[2] = b;
  p.a_rows = g.rows_m;
  p.b_rows = g.rows_n;
  p.k = g.k;
  p.a_ld = g.a.ld;
  p.b_ld = g.b.ld;
  Tl tile;
  tile.init(p, at.m * BM, at.n * BN);
  f32x4 acc[Tl::MT][Tl::NT];
  tile.run(p, 0, 3 * ((g.k + kTileBK - 1) / kTileBK), buf0, buf1, acc);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, wr = wave / WC, wc = wave % WC;
#pragma unroll
  for (int j = 0; j < Tl::NT; ++j) {
    const int n = at.n * BN + (wc * Tl::NT + j) * 16 + (lane & 15);
#pragma unroll
    for (int i = 0; i < Tl::MT; ++i) {
      const int m = at.m * BM + (wr * Tl::MT + i) * 16 + 4 * (lane >> 4);
      if (n >= g.rows_n) {                                  // the transpose's pads
        if (MODE == kUpdate && n < g.out_t.ld) put_column(g.out_t, mat, n, m, g.rows_m, f32x4{0.f, 0.f, 0.f, 0.f});
        continue;
      }
      f32x4 v = acc[i][j] * kDown;                          // times 2^12 of the product
      if constexpr (MODE != kGram) {
        if (m < g.own.ld) v = g.alpha * get_row(g.own, mat, n, m) + g.beta * v;
      }
      if constexpr (kSym) {
        put_row(g.out, mat, n, m, g.rows_m, v);
        if (at.m != at.n) put_column(g.out, mat, n, m, g.rows_m, v);
      } else if constexpr (MODE == kUpdate) {
        put_row(g.out, mat, n, m, g.rows_m, v);
        put_column(g.out_t, mat, n, m, g.rows_m, v);
      } else {
        OT* to = static_cast<OT*>(g.final) + mat * g.final_matrix + n * g.final_ld + m;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          if (m + r >= g.rows_m) break;
          float o = g.scale * kDown * v[r];
          if (g.decay != 0.f) o = fmaf(g.decay, to_f32(to[r]), o);
          to[r] = static_cast<OT>(o);
        }
      }
    }
  }
}

// ---------------------------------------------------------------- host

size_t up256(size_t x) { return (x + 255) & ~static_cast<size_t>(255); }
int64_t up64(int64_t x) { return (x + 63) / 64 * 64; }

struct Layout {
  size_t pieces, x0, t0, x1, t1, a, b, total;
  int m, k;                                 // the smaller and the larger side
  int64_t mp, kp;
  explicit Layout(const umem_orth_desc& od) {
    m = std::min(od.rows, od.cols);
    k = std::max(od.rows, od.cols);
    mp = up64(m);
    kp = up64(k);
    const size_t n = od.n, x = up256(n * 2 * m * kp * 2), t = up256(n * 2 * k * mp * 2), q = up256(n * 2 * m * mp * 2);
    pieces = 0;
    x0 = up256(n * kNormBlocks * sizeof(double));
    t0 = x0 + x;
    x1 = t0 + t;
    t1 = x1 + x;
    a = t1 + t;
    b = a + q;
    total = b + q;
  }
};

Parts parts_at(char* base, size_t at, int rows, int64_t ld) {
  return {reinterpret_cast<uint16_t*>(base + at), rows * ld, ld, 2 * rows * ld};
}

template <Mode MODE, typename OT>
void product(OrthArgs g, int n, hipStream_t s) {
  constexpr bool kSym = MODE == kGram || MODE == kPoly;
#define UMEM_ORTH(BM, WR, WC)                                                                                     \
  {                                                                                                               \
    g.tiles_m = (g.rows_m + BM - 1) / BM;                                                                         \
    g.tiles_n = (g.rows_n + BM - 1) / BM;                                                                         \
    g.items = n * (kSym ? g.tiles_m * (g.tiles_m + 1) / 2 : g.tiles_m * g.tiles_n);                               \
    hipLaunchKernelGGL((orth_product_kernel<MODE, OT, BM, BM, WR, WC>), dim3(tile_grid(g.items)), dim3(64 * WR * WC), \
                       0, s, g);                                                                                  \
  }
  const int64_t large = static_cast<int64_t>(n) * ((g.rows_m + 127) / 128) * ((g.rows_n + 127) / 128);
  if (large >= 512) UMEM_ORTH(128, 2, 2)
  else UMEM_ORTH(64, 2, 2)
#undef UMEM_ORTH
}

template <typename GT>
void first(const umem_orth_desc& od, const GT* g, double* pieces, const Parts& by_rows, const Parts& by_cols,
           hipStream_t s) {
  hipLaunchKernelGGL(orth_norm_kernel<GT>, dim3(kNormBlocks, od.n), dim3(kThreads), 0, s, g,
                     static_cast<int64_t>(od.rows) * od.cols, pieces);
  hipLaunchKernelGGL(orth_first_kernel<GT>, dim3((od.cols + 63) / 64, (od.rows + 63) / 64, od.n), dim3(kThreads), 0, s, g,
                     od.rows, od.cols, od.eps, pieces, by_rows, by_cols);
}

}  // namespace

size_t orth_workspace_bytes(const umem_orth_desc& od) { return Layout(od).total; }

hipError_t launch_orthogonalize(const umem_orth_desc& od, const void* g, void* out, void* ws, hipStream_t s) {
  clear_stale_error();
  const Layout L(od);
  char* base = static_cast<char*>(ws);
  const bool tall = od.rows > od.cols;
  double* pieces = reinterpret_cast<double*>(base + L.pieces);
  // X [m][k] and its transpose, now and next
  Parts x = parts_at(base, L.x0, L.m, L.kp), t = parts_at(base, L.t0, L.k, L.mp);
  Parts x1 = parts_at(base, L.x1, L.m, L.kp), t1 = parts_at(base, L.t1, L.k, L.mp);
  const Parts a = parts_at(base, L.a, L.m, L.mp), b = parts_at(base, L.b, L.m, L.mp);
  if (od.gtype == UMEM_F32) first(od, static_cast<const float*>(g), pieces, tall ? t : x, tall ? x : t, s);
  else first(od, static_cast<const __bf16*>(g), pieces, tall ? t : x, tall ? x : t, s);
  for (int step = 0; step < od.steps; ++step) {
    OrthArgs q{};
    q.a = q.b = x;                                          // A = X X^T
    q.out = a;
    q.rows_m = q.rows_n = L.m;
    q.k = static_cast<int>(L.kp);
    product<kGram, float>(q, od.n, s);
    q.a = q.b = q.own = a;                                  // B = b A + c A^2
    q.out = b;
    q.k = static_cast<int>(L.mp);
    q.alpha = od.b;
    q.beta = od.c;
    product<kPoly, float>(q, od.n, s);
    q.alpha = od.a;                                         // X = a X + B X
    q.beta = 1.f;
    const bool last = step + 1 == od.steps;
    if (!last || !tall) {                                   // m along the larger side
      q.a = t;
      q.b = b;
      q.own = x;
      q.rows_m = L.k;
      q.rows_n = L.m;
      q.out = x1;
      q.out_t = t1;
    } else {
      q.a = b;
      q.b = t;
      q.own = t;
      q.rows_m = L.m;
      q.rows_n = L.k;
    }
    if (!last) {
      product<kUpdate, float>(q, od.n, s);
      std::swap(x, x1);
      std::swap(t, t1);
      continue;
    }
    q.decay = od.decay;
    q.scale = od.scale;
    q.final = out;
    q.final_ld = od.cols;
    q.final_matrix = static_cast<int64_t>(od.rows) * od.cols;
    if (od.otype == UMEM_F32) product<kLast, float>(q, od.n, s);
    else product<kLast, __bf16>(q, od.n, s);
  }
  return hipGetLastError();
}

}  // namespace umem
