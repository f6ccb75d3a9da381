// The orthogonalised update of a matrix by Newton-Schulz products:
//
//   X_0 = G / (|G|_F + eps),  X <- a X + (b A + c A^2) X with A = X X^T,  out = decay out + scale X_steps
//
// on the smaller side: a tall G is worked on transposed, so A is m x m with m = min(rows, cols) <= k.  Every product
// has both operands with k innermost (tiles.h): A's are X's rows, A^2's are A's rows, as A is symmetric, and
// X's update takes B = b A + c A^2 and the transposed X, so X is kept in both orders; of a symmetric product the tiles on and
// below the diagonal are made.  Where k is long, two or three steps are taken on m x m matrices alone, as the steps'
// polynomials commute:
//
//   P = a I + b A + c A^2,  Q <- Q P,  A <- P A P,   then X <- Q X:
//
// 3 products of m x m x m for each step but the first in the place of A = X X^T and B X.  Bounded by the matrix cores for
// large matrices, by the chain of launches for small ones.  Measured, five steps: 896 x 2,048 in 19 launches 191 us, of which
// the 13 products of 896 x 896 x 896 take 9.5 each (one, of two at a time, 12); 1,024 x 16,384 580 us, X X^T 52 + 9 (36 of 64 tiles, three pairs of
// parts: 1.1 PFLOP/s), X's update 123, 0.84 PFLOP/s.
//
// Rounding: every matrix between the steps is two fp16 parts of its values times a power of two (2^12; 2^9 for P and Q),
// which hold 22 bits of it, and a product takes three of the four pairs of parts (the fourth is below 2^-22 of the
// result); sums are fp32, |G|_F is fp64.  Two bf16 parts would hold 17 bits: what a step loses of X's small singular
// values grows by a = 3.4 a step.  After five steps of a random 448 x 1,792 matrix one step at a time is 6e-7 off the
// exact result, two and three at a time 7e-7, the bf16 parts 4e-5, fp32 throughout 1e-6; of one with a direction 100 times as
// strong as the others 5e-6, 1e-5 and, in fp32, 1e-5.
// An entry of X, A or B that reaches 16, of Q 128, becomes infinite: of coefficients that keep singular values of 1
// near 1 none does.
#include <algorithm>
#include <cmath>

#include "tiles.h"

namespace umem {
namespace {

constexpr int kThreads = 256;
constexpr int kUpBits = 12;
constexpr float kDown = 1.f / (1 << kUpBits);

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

// A matrix whose rows hold ld elements: both parts of ld / 2 values (part_at); how far the next matrix of the batch is.
struct Parts {
  uint16_t* p;
  int64_t ld, matrix;
};

// Eight words to a row of both parts.
__device__ __forceinline__ void put_eight(const Parts& out, int64_t mat, int row, int at, const uint32_t (&w)[8]) {
  uint16_t* to = out.p + mat * out.matrix + row * out.ld + part_at(at);
  *reinterpret_cast<u32x4*>(to) = u32x4{(w[0] & 0xffffu) | w[1] << 16, (w[2] & 0xffffu) | w[3] << 16,
                                        (w[4] & 0xffffu) | w[5] << 16, (w[6] & 0xffffu) | w[7] << 16};
  *reinterpret_cast<u32x4*>(to + kPartStep) = u32x4{w[0] >> 16 | (w[1] & 0xffff0000u), w[2] >> 16 | (w[3] & 0xffff0000u),
                                                    w[4] >> 16 | (w[5] & 0xffff0000u), w[6] >> 16 | (w[7] & 0xffff0000u)};
}

// ---------------------------------------------------------------- norm and first X

// Workgroups that a matrix's norm is spread over: 4,096 elements or more each.
int norm_blocks(const umem_orth_desc& od) {
  return static_cast<int>(std::min<int64_t>(512, (static_cast<int64_t>(od.rows) * od.cols + 4095) / 4096));
}

// |G|^2 of each matrix, in fp64 pieces of fixed ranges.
template <typename T>
__global__ __launch_bounds__(kThreads) void orth_norm_kernel(const T* __restrict__ g, int64_t size,
                                                             double* __restrict__ pieces) {
  typedef T four __attribute__((ext_vector_type(4), aligned(sizeof(T))));
  __shared__ double waves[kThreads / kWave];
  const T* m = g + blockIdx.y * size;
  const int64_t step = static_cast<int64_t>(gridDim.x) * kThreads * 4;
  double sum[4] = {0.0, 0.0, 0.0, 0.0};
  int64_t i = (static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x) * 4;
#pragma unroll 4
  for (; i + 4 <= size; i += step) {
    const four v = *reinterpret_cast<const four*>(m + i);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const double x = to_f32(v[j]);
      sum[j] = fma(x, x, sum[j]);
    }
  }
  for (; i < size && (i & 3) != 3; ++i) {                   // the last, partial four
    const double x = to_f32(m[i]);
    sum[0] = fma(x, x, sum[0]);
  }
  double all = (sum[0] + sum[1]) + (sum[2] + sum[3]);
#pragma unroll
  for (int off = kWave / 2; off > 0; off >>= 1) all += __shfl_xor(all, off, kWave);
  if ((threadIdx.x & (kWave - 1)) == 0) waves[threadIdx.x / kWave] = all;
  __syncthreads();
  if (threadIdx.x == 0) {
#pragma unroll
    for (int w = 1; w < kThreads / kWave; ++w) all += waves[w];
    pieces[blockIdx.y * gridDim.x + blockIdx.x] = all;
  }
}

// X_0 in both orders, with zeros up to the rows' ends; a 64 x 64 tile of G a workgroup.  by_rows [rows][ld of cols],
// by_cols [cols][ld of rows].
template <typename T>
__global__ __launch_bounds__(kThreads) void orth_first_kernel(const T* __restrict__ g, int rows, int cols, float eps,
                                                              const double* __restrict__ pieces, int blocks,
                                                              Parts by_rows, Parts by_cols) {
  __shared__ uint32_t tile[64][65];
  const int r0 = blockIdx.y * 64, c0 = blockIdx.x * 64, c = threadIdx.x % 64;
  const int64_t mat = blockIdx.z;
  const T* m = g + mat * rows * static_cast<int64_t>(cols) + min(c0 + c, cols - 1);
  float v[16];                                              // all under way before the first is waited for
#pragma unroll
  for (int i = 0; i < 16; ++i)
    v[i] = to_f32(m[min(r0 + i * 4 + static_cast<int>(threadIdx.x / 64), rows - 1) * static_cast<int64_t>(cols)]);
  double sum = 0.0;                                         // every wave adds the pieces for itself
#pragma unroll 8
  for (int i = threadIdx.x & (kWave - 1); i < blocks; i += kWave) sum += pieces[mat * blocks + i];
#pragma unroll
  for (int off = kWave / 2; off > 0; off >>= 1) sum += __shfl_xor(sum, off, kWave);
  int e = 0;                                                // (the norm of values within fp32 may be past it)
  const float norm = static_cast<float>(frexp(sqrt(sum) + static_cast<double>(eps), &e));
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const int r = i * 4 + threadIdx.x / 64;
    uint32_t hi, lo;
    f16_parts(ldexpf(v[i], kUpBits - e) / norm, hi, lo);
    tile[r][c] = r0 + r < rows && c0 + c < cols ? hi | lo << 16 : 0u;
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int a = i * 32 + threadIdx.x / 8, b = (threadIdx.x % 8) * 8;
    uint32_t w[8];
    if (r0 + a < rows) {
#pragma unroll
      for (int j = 0; j < 8; ++j) w[j] = tile[a][b + j];
      put_eight(by_rows, mat, r0 + a, c0 + b, w);
    }
    if (c0 + a < cols) {
#pragma unroll
      for (int j = 0; j < 8; ++j) w[j] = tile[b + j][a];
      put_eight(by_cols, mat, c0 + a, r0 + b, w);
    }
  }
}

// ---------------------------------------------------------------- products

// A = X X^T; B = b A + c A^2; P = a I + B; a product of two polynomials of A (Q P, P A); X = a X + B X, or Q X; the same
// into the output.
enum Mode { kGram, kPoly, kShifted, kTimes, kUpdate, kApply, kLast, kLastApply };
constexpr bool symmetric(Mode m) { return m == kGram || m == kPoly || m == kShifted || m == kTimes; }
constexpr bool has_own(Mode m) { return m == kPoly || m == kShifted || m == kUpdate || m == kLast; }
constexpr bool is_last(Mode m) { return m == kLast || m == kLastApply; }
constexpr bool is_update(Mode m) { return m == kUpdate || m == kApply; }
// P and Q are held times 2^9.  The sums of a product hold both its operands' powers, its result one of them.
constexpr float kDownQ = 1.f / 512.f;
constexpr float down(Mode m) { return m == kTimes || m == kApply || m == kLastApply ? kDownQ : kDown; }

struct OrthArgs {
  Parts a, b;             // the product's operands: rows along m and along n, k innermost
  Parts own;              // kPoly, kShifted: A; kUpdate, kLast: X by rows n, m along its rows
  Parts out, out_t;       // the product (symmetric), or X by rows n and, in out_t, transposed
  Parts a2, b2, out2;     // a second symmetric product of the same shape (jobs == 2)
  int jobs;
  int rows_m, rows_n;
  int k;                  // elements of a row that the product walks
  int tiles_m, tiles_n, per, items;        // of a matrix: tiles; of all matrices: items
  int splits;             // parts of k, each an item of its own with its sums to partial [split][item][BN][BM]
  float* partial;
  float alpha, beta;      // with own: alpha own + beta product
  float shift;            // kShifted: added to the diagonal
  float decay, scale;     // the last X: final = decay final + scale X, [n][m] of final_ld
  void* final;
  int64_t final_ld, final_matrix;
};

// The matrix and the tile of an item; of a symmetric product the tiles with n <= m alone.
struct OrthTile {
  int64_t mat;
  int m, n;
};
template <Mode MODE>
__device__ __forceinline__ OrthTile orth_tile(const OrthArgs& g, int item) {
  const int mat = item / g.per, in = item - mat * g.per;
  if constexpr (!symmetric(MODE)) {
    const TilePlace at = tile_place(in, g.tiles_m, g.tiles_n);
    return {mat, at.m, at.n};
  }
  int m = static_cast<int>((sqrtf(8.f * in + 1.f) - 1.f) * 0.5f);
  while ((m + 1) * (m + 2) / 2 <= in) ++m;
  while (m * (m + 1) / 2 > in) --m;
  return {mat, m, in - m * (m + 1) / 2};
}

// The four values at row n, columns m .. m + 3.
__device__ __forceinline__ f32x4 get_four(const Parts& in, int64_t mat, int n, int m) {
  const uint16_t* from = in.p + mat * in.matrix + n * in.ld + part_at(m);
  const u32x2 hi = *reinterpret_cast<const u32x2*>(from), lo = *reinterpret_cast<const u32x2*>(from + kPartStep);
  return f32x4{bits_f32(hi.x & 0xffffu) + bits_f32(lo.x & 0xffffu), bits_f32(hi.x >> 16) + bits_f32(lo.x >> 16),
               bits_f32(hi.y & 0xffffu) + bits_f32(lo.y & 0xffffu), bits_f32(hi.y >> 16) + bits_f32(lo.y >> 16)};
}

// A product's four sums at (n, m .. m + 3) become four values of the result with their two parts in a word each, zeros
// past the matrix; or go to the final output.
template <Mode MODE, typename OT>
__device__ __forceinline__ u32x4 finish_four(const OrthArgs& g, int64_t mat, int n, int m, f32x4 v) {
  const bool in = n < g.rows_n && m < g.rows_m;
  v *= down(MODE);
  if constexpr (has_own(MODE)) {
    if (in) v = g.alpha * get_four(g.own, mat, n, m) + g.beta * v;
  }
  if constexpr (MODE == kShifted) {
    v *= kDown / kDownQ;
#pragma unroll
    for (int r = 0; r < 4; ++r) v[r] += m + r == n ? g.shift / kDownQ : 0.f;
  }
  if constexpr (is_last(MODE)) {
    if (!in) return u32x4{0u, 0u, 0u, 0u};
    OT* to = static_cast<OT*>(g.final) + mat * g.final_matrix + n * g.final_ld + m;
    v *= kDown;                           // (not as a part of the scale, which may be as small as fp32 holds)
    typedef OT four __attribute__((ext_vector_type(4), aligned(sizeof(OT))));
    if (m + 4 <= g.rows_m) {
      four o;
      if (g.decay != 0.f) {
        const four h = *reinterpret_cast<const four*>(to);
#pragma unroll
        for (int r = 0; r < 4; ++r) o[r] = static_cast<OT>(fmaf(g.decay, to_f32(h[r]), g.scale * v[r]));
      } else {
#pragma unroll
        for (int r = 0; r < 4; ++r) o[r] = static_cast<OT>(g.scale * v[r]);
      }
      *reinterpret_cast<four*>(to) = o;
    } else {
#pragma unroll
      for (int r = 0; r < 3; ++r) {
        if (m + r >= g.rows_m) break;
        to[r] = static_cast<OT>(g.decay != 0.f ? fmaf(g.decay, to_f32(to[r]), g.scale * v[r]) : g.scale * v[r]);
      }
    }
    return u32x4{0u, 0u, 0u, 0u};
  }
  u32x4 w;
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    uint32_t hi, lo;
    f16_parts(v[r], hi, lo);
    w[r] = in && m + r < g.rows_m ? hi | lo << 16 : 0u;
  }
  return w;
}

// A block of 64 x BM words in LDS, [n][m]; a row's 16-byte pieces are permuted by its number, so that rows and
// columns are both read without meeting in a bank.
template <int BM>
__device__ __forceinline__ int word_at(int n, int m) {
  return n * BM + ((((m >> 2) ^ n) & (BM / 4 - 1)) << 2) + (m & 3);
}


// The block of the result at (m0, n0) from LDS to memory, by rows and (or of a symmetric result the mirrored tile) by
// columns.
template <Mode MODE, int BM, int BN, int THREADS, typename At>
__device__ __forceinline__ void put_block(const OrthArgs& g, const Parts& rows, int64_t mat, int m0, int n0, bool mirrored, const At& word) {
  for (int i = threadIdx.x; i < BN * (BM / 8); i += THREADS) {
    const int n = i / (BM / 8), m = (i % (BM / 8)) * 8;
    if (n0 + n >= g.rows_n || 2 * (m0 + m) >= rows.ld) continue;
    uint32_t w[8];
    *reinterpret_cast<u32x4*>(w) = *reinterpret_cast<const u32x4*>(word(n, m));
    *reinterpret_cast<u32x4*>(w + 4) = *reinterpret_cast<const u32x4*>(word(n, m + 4));
    put_eight(rows, mat, n0 + n, m0 + m, w);
  }
  if (!is_update(MODE) && !mirrored) return;
  const Parts& out = is_update(MODE) ? g.out_t : rows;
  // eight lanes (of 32 columns four) to 64 consecutive n of a column, eight columns together
  constexpr int kPieces = BN < 64 ? BN / 8 : 8;
  for (int i = threadIdx.x; i < BM * (BN / 8); i += THREADS) {
    const int group = i / (8 * kPieces), m = (group % (BM / 8)) * 8 + (i & 7);
    const int n = (group / (BM / 8)) * 64 + ((i >> 3) % kPieces) * 8;
    if (m0 + m >= g.rows_m || 2 * (n0 + n) >= out.ld) continue;
    uint32_t w[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) w[j] = *word(n + j, m);
    put_eight(out, mat, m0 + m, n0 + n, w);
  }
}

template <Mode MODE, typename OT, int BM, int BN, int WR, int WC, int BUFS, int GROUPS>
__global__ __launch_bounds__(64 * WR * WC * GROUPS) __attribute__((amdgpu_waves_per_eu(BN == 64 && GROUPS == 1 ? 3 : 2))) void orth_product_kernel(OrthArgs g) {
  typedef Tile<true, BM, BN, WR, WC, BUFS, kBoth, GROUPS> Tl;
  constexpr int kLds = GROUPS * Tl::kElems, kHalves = BM / BN;
  static_assert(BN <= 64 ? 2 * BM * BN <= kLds : BN % 128 == 0 && BM * BN <= Tl::kElems,
                "a tile of words fits the operands' LDS");
  __shared__ __align__(16) uint16_t buf0[kLds];
  __shared__ __align__(16) uint16_t buf1[kLds];
  __shared__ __align__(16) uint16_t buf2[BUFS > 2 ? kLds : 8];
  __shared__ __align__(16) uint16_t buf3[BUFS > 3 ? kLds : 8];
  const int all = g.items * g.splits * g.jobs, id = tile_item(all);
  if (id >= all) return;                                    // the whole workgroup: no barrier is skipped
  const int split = id / g.items, item = id - split * g.items;          // or of two products which one
  const bool second = MODE == kTimes && g.jobs == 2 && split == 1;
  const OrthTile at = orth_tile<MODE>(g, item / kHalves);
  const int m0 = at.m * BM, n0 = at.n * BM + item % kHalves * BN;
  TilePairs p;
  p.n = 1;
  p.a[0] = (second ? g.a2.p : g.a.p) + at.mat * g.a.matrix;
  p.b[0] = (second ? g.b2.p : g.b.p) + at.mat * g.b.matrix;
  p.a_rows = g.rows_m;
  p.b_rows = g.rows_n;
  p.k = g.k;
  p.a_ld = g.a.ld;
  p.b_ld = g.b.ld;
  Tl tile;
  tile.init(p, m0, n0);
  f32x4 acc[Tl::MT][Tl::NT];
  const int64_t slices = Tl::slices(p);
  const int part = g.jobs == 2 ? 0 : split;
  const int from = static_cast<int>(slices * part / g.splits), to = static_cast<int>(slices * (part + 1) / g.splits);
  const int group = Tl::group(), mine = group * Tl::kElems;
  tile.run(p, from, to, buf0 + mine, buf1 + mine, buf2 + (BUFS > 2 ? mine : 0), buf3 + (BUFS > 3 ? mine : 0), acc);
  const int lane = threadIdx.x & 63, wave = Tl::thread() >> 6, wr = wave / WC, wc = wave % WC;
  const int m_in = wr * Tl::MT * 16 + 4 * (lane >> 4), n_in = wc * Tl::NT * 16 + (lane & 15);
  // Of several groups each ends a share of the tile's blocks, the sums of all of them in their order.
  constexpr int kBlocks = Tl::MT * Tl::NT, kOwn = kBlocks / GROUPS;
  f32x4 sum[kOwn];
  if constexpr (GROUPS > 1) {
    static_assert(kBlocks % GROUPS == 0 && BM * BN * 4 <= Tl::kElems * 2, "a group's blocks fit its part of a buffer");
    f32x4* sums = reinterpret_cast<f32x4*>(buf1) + Tl::thread();
    __syncthreads();
#pragma unroll
    for (int o = 0; o < kBlocks; ++o) sums[(group * kBlocks + o) * Tl::kThreads] = acc[o % Tl::MT][o / Tl::MT];
    __syncthreads();
#pragma unroll
    for (int o = 0; o < kOwn; ++o) {
      sum[o] = sums[(group * kOwn + o) * Tl::kThreads];
#pragma unroll
      for (int i = 1; i < GROUPS; ++i) sum[o] += sums[(i * kBlocks + group * kOwn + o) * Tl::kThreads];
    }
  } else {
#pragma unroll
    for (int o = 0; o < kOwn; ++o) sum[o] = acc[o % Tl::MT][o / Tl::MT];
  }
  const auto m_of = [&](int o) { return m_in + (GROUPS == 1 ? o : group * kOwn + o) % Tl::MT * 16; };
  const auto n_of = [&](int o) { return n_in + (GROUPS == 1 ? o : group * kOwn + o) / Tl::MT * 16; };
  if (MODE == kGram && g.splits > 1) {
    float* to = g.partial + static_cast<int64_t>(id) * (BM * BN);
#pragma unroll
    for (int o = 0; o < kOwn; ++o) *reinterpret_cast<f32x4*>(to + n_of(o) * BM + m_of(o)) = sum[o];
    return;
  }
  const auto word = [&](int n, int m) {
    uint16_t* half = BN <= 64 || n < BN / 2 ? buf0 : buf1;
    return reinterpret_cast<uint32_t*>(half) + word_at<BM>(BN <= 64 ? n : n % (BN / 2), m);
  };
  if (!is_last(MODE) && GROUPS == 1) __syncthreads();       // the last slice has been read
#pragma unroll
  for (int o = 0; o < kOwn; ++o) {
    const u32x4 w = finish_four<MODE, OT>(g, at.mat, n0 + n_of(o), m0 + m_of(o), sum[o]);
    if (!is_last(MODE)) *reinterpret_cast<u32x4*>(word(n_of(o), m_of(o))) = w;
  }
  if (is_last(MODE)) return;
  __syncthreads();
  put_block<MODE, BM, BN, Tl::kThreads * GROUPS>(g, second ? g.out2 : g.out, at.mat, m0, n0, at.m != at.n, word);
}

// The sums of the splits of X X^T, in their order; a 64 x 64 block of a tile a workgroup.
template <int BM>
__global__ __launch_bounds__(kThreads) void orth_join_kernel(OrthArgs g) {
  __shared__ __align__(16) uint32_t words[64 * 64];
  constexpr int kSub = BM / 64;
  const int item = blockIdx.x / (kSub * kSub), sub = blockIdx.x % (kSub * kSub);
  const OrthTile at = orth_tile<kGram>(g, item);
  const int m_in = (sub % kSub) * 64, n_in = (sub / kSub) * 64;
  const int m0 = at.m * BM + m_in, n0 = at.n * BM + n_in;
  if (m0 >= g.rows_m || n0 >= g.rows_n) return;
  const float* from = g.partial + static_cast<int64_t>(item) * (BM * BM);
  const int64_t next = static_cast<int64_t>(g.items) * (BM * BM);
  const auto word = [&](int n, int m) { return words + word_at<64>(n, m); };
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int n = (threadIdx.x >> 4) + i * 16, m = (threadIdx.x & 15) * 4;
    const float* q = from + (n_in + n) * BM + m_in + m;
    f32x4 v = *reinterpret_cast<const f32x4*>(q);
#pragma unroll 4
    for (int s = 1; s < g.splits; ++s) v += *reinterpret_cast<const f32x4*>(q + s * next);
    *reinterpret_cast<u32x4*>(word(n, m)) = finish_four<kGram, float>(g, at.mat, n0 + n, m0 + m, v);
  }
  __syncthreads();
  put_block<kGram, 64, 64, kThreads>(g, g.out, at.mat, m0, n0, at.m != at.n, word);
}

// ---------------------------------------------------------------- host

size_t up256(size_t x) { return (x + 255) & ~static_cast<size_t>(255); }
int64_t up64(int64_t x) { return (x + 63) / 64 * 64; }

// A product's tiles and how often k is split, by what both sizes of tile measured (us; slices of 32 values):
// a 64 x 64 tile (3 buffers, 3 workgroups a CU) takes 0.25 a slice alone on its CU, 0.4 and 0.6 beside one and two
// others; a 128 x 128 tile (eight waves, 4 buffers, a CU to itself) 0.47.  So 64 x 64 wins where tiles are few and
// k is short: 896 x 896 x 896 of A^2 11 and 23, of 2,048 x 2,048 x 2,048 42 and 44; 128 x 128 where there are many: 1,024 x
// 16,384 of X 141 and 126, 2,048 x 8,192 240 and 210.  A split's partial sums and the launch that adds them take 4 or more: 896
// x 896 over 2,048 20.7 in one piece, 17.0 in two, 18.6 in four; 1,024 x 1,024 over 16,384 242 in one, 60 in six.
struct Plan {
  int bm, splits;
  double us;
  bool halves;            // a workgroup takes half a tile, with four groups of waves: 896 x 896 x 896 11.0 -> 9.5 us
  bool alone;             // every workgroup has a CU to itself: two groups of waves share its slices (four with two buffers
                          // each 1.15 times as long; two where two workgroups share a CU, or four buffers, the same)
};
constexpr int kMostSplits = 16, kCus = 256;
constexpr size_t kPartialBytes = size_t{64} << 20;
int64_t tile_count(int bm, int n, int rows_m, int rows_n, bool sym) {
  const int64_t tm = (rows_m + bm - 1) / bm, tn = (rows_n + bm - 1) / bm;
  return n * (sym ? tm * (tm + 1) / 2 : tm * tn);
}
Plan plan(int n, int rows_m, int rows_n, int slices, bool sym, int jobs = 1, int most_splits = 1) {
  Plan best{64, 1, 1e300, false, false};
  for (int bm : {64, 128}) {
    const int64_t it = tile_count(bm, n, rows_m, rows_n, sym);
    for (int s = 1; s <= most_splits && s <= slices; ++s) {
      const double bytes = static_cast<double>(it) * s * bm * bm * sizeof(float);
      if (s > 1 && bytes > kPartialBytes) break;
      const int64_t wgs = it * s * jobs, cus = (wgs + kCus - 1) / kCus;          // workgroups of the fullest CU
      const double each = (slices + s - 1) / s;
      double cost = s > 1 ? 4.5 + 0.7 * s + bytes / 2.5e6 : 0.0;
      const bool halves = sym && bm == 64 && s == 1 && 2 * wgs <= kCus && each >= 8;
      if (bm == 128) {
        cost += static_cast<double>(cus) * (3.0 + 0.47 * each);
      } else {
        const int rest = static_cast<int>(cus % 3);
        cost += static_cast<double>(cus / 3) * (3.0 + 0.6 * each);
        if (rest) cost += 3.0 + (halves ? 0.1 : cus == 1 ? 0.15 : rest == 1 ? 0.25 : 0.4) * each;
      }
      if (cost < best.us) best = {bm, s, cost, halves, bm == 64 && cus == 1 && each >= 4};
    }
  }
  return best;
}

// Of X X^T, whose k is the longer side; the other products' k is the shorter one, and a split of it never pays.
Plan plan_gram(int n, int m, int slices) { return plan(n, m, m, slices, true, 1, kMostSplits); }
size_t partial_bytes(int n, int m, int slices) {
  const Plan p = plan_gram(n, m, slices);
  return p.splits == 1 ? 0 : up256(tile_count(p.bm, n, m, m, true) * p.splits * p.bm * p.bm * sizeof(float));
}

// How the steps are taken: one at a time (rounds == steps), or in rounds of two or three on m x m matrices, where that
// is less time and G is at least twice as long as wide.  A round loses more of what is small against the largest singular
// value.  Five steps, by 3 and 2, are 0.7 to 2.5 times as far from the exact result as fp32 one at a time (300 x 2,000: flat
// and steep spectra 3e-6 and 2e-6 off, rank 1 8e-5; one at a time 0.3 to 1 times), but a square random matrix, whose
// smallest singular value is next to none, would be 4 times.  Three steps of rank 1 are 4e-5 off (fp32 1e-5), and of 16 steps
// a flat spectrum 5e-5 (7e-6); rows that are there twice, whose zeros fp32 keeps by chance, 9e-5 in 8 steps (2e-6).
// fp32 in the same rounds loses as much or more.
struct Steps {
  int rounds;
  int of(int round, int steps) const { return steps / rounds + (round < steps % rounds ? 1 : 0); }     // the longer ones first
};
Steps plan_steps(const umem_orth_desc& od, int m, int k) {
  const int n = od.n, xs = static_cast<int>(up64(k) / 32), as = static_cast<int>(up64(m) / 32);
  int most = 3;                                             // Q stays below 128: a^3 = 41 of the usual coefficients
  while (most > 1 && std::pow(std::fabs(od.a), most) > 100.f) --most;
  if (most == 1 || k < 2 * m) return {od.steps};
  const double one = plan_gram(n, m, xs).us + plan(n, k, m, as, false).us;
  const double two = plan(n, m, m, as, true, 2).us + plan(n, m, m, as, true).us;
  return {two < one ? (od.steps + most - 1) / most : od.steps};
}

struct Layout {
  size_t pieces, x0, t0, x1, t1, q, partial, total;
  size_t square;                            // a matrix of m x m: A, B or P, and in rounds Q (two) and T
  int m, k;                                 // the smaller and the larger side
  int64_t mp, kp;                           // values of a row
  Steps steps;
  explicit Layout(const umem_orth_desc& od) {
    m = std::min(od.rows, od.cols);
    k = std::max(od.rows, od.cols);
    mp = up64(m);
    kp = up64(k);
    steps = plan_steps(od, m, k);
    const size_t n = od.n, x = up256(n * 4 * m * kp), t = up256(n * 4 * k * mp);
    square = up256(n * 4 * m * mp);
    pieces = 0;
    x0 = up256(n * norm_blocks(od) * sizeof(double));
    t0 = x0 + x;
    x1 = t0 + t;
    t1 = x1 + x;
    q = t1 + t;
    partial = q + (steps.rounds < od.steps ? 5 : 2) * square;
    total = partial + partial_bytes(od.n, m, static_cast<int>(kp / 32));
  }
};

Parts parts_at(char* base, size_t at, int rows, int64_t values) {
  return {reinterpret_cast<uint16_t*>(base + at), 2 * values, 2 * rows * values};
}

template <Mode MODE, typename OT = float>
void product(OrthArgs g, int n, hipStream_t s) {
  g.jobs = std::max(g.jobs, 1);
  const Plan pl = MODE == kGram ? plan_gram(n, g.rows_m, g.k / kTileBK)
                                : plan(n, g.rows_m, g.rows_n, g.k / kTileBK, symmetric(MODE), g.jobs);
  g.splits = pl.splits;
  constexpr int kHalf = symmetric(MODE) ? 32 : 64;          // (the others have no halves, and no instance of their own)
#define UMEM_ORTH(BM, BN, WR, WC, BUFS, GROUPS)                                                                      \
  {                                                                                                                  \
    g.tiles_m = (g.rows_m + BM - 1) / BM;                                                                            \
    g.tiles_n = (g.rows_n + BM - 1) / BM;                                                                            \
    g.per = symmetric(MODE) ? g.tiles_m * (g.tiles_m + 1) / 2 : g.tiles_m * g.tiles_n;                               \
    g.items = n * g.per * (BM / BN);                                                                                 \
    hipLaunchKernelGGL((orth_product_kernel<MODE, OT, BM, BN, WR, WC, BUFS, GROUPS>),                                \
                       dim3(tile_grid(g.items * g.splits * g.jobs)), dim3(64 * WR * WC * GROUPS), 0, s, g);          \
    if (MODE == kGram && g.splits > 1)                                                                               \
      hipLaunchKernelGGL(orth_join_kernel<BM>, dim3(g.items * (BM / 64) * (BM / 64)), dim3(kThreads), 0, s, g);      \
  }
  if (pl.bm == 128) UMEM_ORTH(128, 128, 4, 2, 4, 1)
  else if (symmetric(MODE) && pl.halves) UMEM_ORTH(64, kHalf, 2, kHalf / 32, 3, 128 / kHalf)
  else if (pl.alone) UMEM_ORTH(64, 64, 2, 2, 3, 2)
  else UMEM_ORTH(64, 64, 2, 2, 3, 1)
#undef UMEM_ORTH
}

template <typename GT>
void first(const umem_orth_desc& od, const GT* g, double* pieces, const Parts& by_rows, const Parts& by_cols,
           hipStream_t s) {
  hipLaunchKernelGGL(orth_norm_kernel<GT>, dim3(norm_blocks(od), od.n), dim3(kThreads), 0, s, g,
                     static_cast<int64_t>(od.rows) * od.cols, pieces);
  hipLaunchKernelGGL(orth_first_kernel<GT>, dim3((od.cols + 63) / 64, (od.rows + 63) / 64, od.n), dim3(kThreads), 0, s, g,
                     od.rows, od.cols, od.eps, pieces, norm_blocks(od), by_rows, by_cols);
}

}  // namespace

size_t orth_workspace_bytes(const umem_orth_desc& od) {
  return std::min(od.rows, od.cols) <= kMaxOrthSmall ? orth_small_workspace_bytes(od) : Layout(od).total;
}

hipError_t launch_orthogonalize(const umem_orth_desc& od, const void* g, void* out, void* ws, hipStream_t s) {
  if (std::min(od.rows, od.cols) <= kMaxOrthSmall) return launch_orth_small(od, g, out, ws, s);
  clear_stale_error();
  const Layout L(od);
  char* base = static_cast<char*>(ws);
  const bool tall = od.rows > od.cols;
  double* pieces = reinterpret_cast<double*>(base + L.pieces);
  // X [m][k] and its transpose, now and next
  Parts x = parts_at(base, L.x0, L.m, L.kp), t = parts_at(base, L.t0, L.k, L.mp);
  Parts x1 = parts_at(base, L.x1, L.m, L.kp), t1 = parts_at(base, L.t1, L.k, L.mp);
  const auto square = [&](int i) { return parts_at(base, L.q + i * L.square, L.m, L.mp); };
  Parts a = square(0), q = square(1), q1 = square(2);
  const Parts p = square(3), w = square(4);
  if (od.gtype == UMEM_F32) first(od, static_cast<const float*>(g), pieces, tall ? t : x, tall ? x : t, s);
  else first(od, static_cast<const __bf16*>(g), pieces, tall ? t : x, tall ? x : t, s);
  OrthArgs sq{};                                            // m x m of rows of A
  sq.partial = reinterpret_cast<float*>(base + L.partial);
  sq.rows_m = sq.rows_n = L.m;
  sq.k = static_cast<int>(a.ld);
  for (int round = 0; round < L.steps.rounds; ++round) {
    const int steps = L.steps.of(round, od.steps);
    OrthArgs o = sq;
    o.a = o.b = x;                                          // A = X X^T
    o.out = a;
    o.k = static_cast<int>(x.ld);
    product<kGram>(o, od.n, s);
    for (int step = 0; step < steps; ++step) {
      o = sq;
      o.a = o.b = o.own = a;
      o.alpha = od.b;
      o.beta = od.c;
      if (steps == 1) {                                     // B = b A + c A^2
        o.out = q;
        product<kPoly>(o, od.n, s);
        break;
      }
      o.shift = od.a;                                       // P = a I + b A + c A^2
      o.out = step == 0 ? q : p;
      product<kShifted>(o, od.n, s);
      const bool end = step + 1 == steps;
      o = sq;
      if (!end) {                                           // T = P A
        o.a = step == 0 ? q : p;
        o.b = a;
        o.out = w;
      }
      if (step > 0) {                                       // Q = Q P
        (end ? o.a : o.a2) = q;
        (end ? o.b : o.b2) = p;
        (end ? o.out : o.out2) = q1;
        o.jobs = end ? 1 : 2;
      }
      if (!end || step > 0) product<kTimes>(o, od.n, s);
      if (step > 0) std::swap(q, q1);
      if (end) break;
      o = sq;                                               // A = P T
      o.a = step == 0 ? q : p;
      o.b = w;
      o.out = a;
      product<kTimes>(o, od.n, s);
    }
    const bool last = round + 1 == L.steps.rounds;
    const bool turned = last && tall;                       // the last X goes out as G lies
    o = sq;
    o.a = turned ? q : t;                                   // X = a X + B X, or Q X
    o.b = turned ? t : q;
    o.own = turned ? t : x;
    o.alpha = od.a;
    o.beta = 1.f;
    o.rows_m = turned ? L.m : L.k;
    o.rows_n = turned ? L.k : L.m;
    if (!last) {
      o.out = x1;
      o.out_t = t1;
      if (steps == 1) product<kUpdate>(o, od.n, s);
      else product<kApply>(o, od.n, s);
      std::swap(x, x1);
      std::swap(t, t1);
      continue;
    }
    o.decay = od.decay;
    o.scale = od.scale;
    o.final = out;
    o.final_ld = od.cols;
    o.final_matrix = static_cast<int64_t>(od.rows) * od.cols;
    if (od.otype == UMEM_F32) {
      if (steps == 1) product<kLast, float>(o, od.n, s);
      else product<kLastApply, float>(o, od.n, s);
    } else {
      if (steps == 1) product<kLast, __bf16>(o, od.n, s);
      else product<kLastApply, __bf16>(o, od.n, s);
    }
  }
  return hipGetLastError();
}

}  // namespace umem
