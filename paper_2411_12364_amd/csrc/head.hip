// The head of a model: softmax cross entropy of a large vocabulary from the hidden states, and its gradients, without
// the logits ever being kept.
//
//   z[t][v] = s <x[t], W[v]>,  lse[t] = log sum_v exp z[t][v],  loss[t] = lse[t] - z[t][y[t]]
//   r[t][v] = s dloss[t] (exp(z[t][v] - lse[t]) - [v = y[t]]),  dx = r W,  dW (+)= r^T x
//
// Forward: tiles of logits (tiles.h; the vocabulary along m) are made on the matrix cores and reduced where
// they are, in registers, to each token's maximum and sum of exponentials over the tile's rows; a second kernel joins the
// tiles' pairs in their order.  Backward: the vocabulary goes by pieces; for each the logits are made again, r goes to
// scratch in bf16 in both orders, and two more products take it, all three with k innermost (x and the piece's rows of
// W are laid out transposed beforehand).  Bounded by the matrix cores: 2 T V d operations forward, 6 T V d backward, but
// for few tokens, where W is read once at the rate of the memory.  Measured: 16 tokens by 50,000 rows of 2,048 40 + 5 us (W
// at 5.2 TB/s); 8,192 tokens by 50,000 of 2,048, forward and backward with dW in fp32, 7.5 ms for 8.3 TFLOP: the logits 1.33 ms
// (1.25 PFLOP/s), then for each 7,168 rows r 252 us, W's transpose 11, dx 207 (1.14 PFLOP/s), dW 399 (two products, 1.18).
// Tokens that do not count are left out of the backward: a list of those that do is made first, and every product's grid and
// length follow its count on the device (2,000 tokens, a third of them without a target, by 32,003 of 1,024 642 us with
// them, so 528).
//
// Rounding: logits and sums are fp32 of bf16 operands; fp32 x is three bf16 parts, which hold it whole.  r is made for
// losses' gradients of at most 1, and the largest of them and s are multiplied in last, in fp32: the gradient of a
// mean has one value for all tokens, and a target's r of nearly that value times -s would be rounded the same way
// for all of them.  For dx r is bf16 beside W: one part where dx is bf16 (both roundings are of the result's own
// size), three, which hold it whole, where it is fp32.  For dW r and x are fp16, r times 2^15 and x times the power
// of two that takes its largest value to that: a bf16 x down to 2^-32 of the largest is held whole, and r as
// one part (2^-12 of it, and 2^-40 of the largest dloss) where dW is bf16, as two (22 bits) where it is fp32, as fp32 x is then.
// (Three bf16 parts of r hold it as well, at half more time: 8,192 tokens by 7,168 rows of 2,048 560 us, so 370.)
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "tiles.h"

namespace umem {
namespace {

constexpr int kThreads = 256;

__device__ __forceinline__ uint32_t bf16_bits(float x) {
  return __builtin_bit_cast(uint16_t, static_cast<__bf16>(x));
}
__device__ __forceinline__ float bits_f32(uint32_t b) { return __uint_as_float(b << 16); }

// Part `part` of x as a sum of bf16 parts.  What is past the first part of a value that is no number, or too large for
// bf16, is zero.
template <int N>
__device__ __forceinline__ void bf16_parts(float x, uint32_t (&p)[N]) {
  float rest = x;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    p[i] = bf16_bits(rest);
    const float v = bits_f32(p[i]);
    rest = fabsf(v) <= 3.4e38f ? rest - v : 0.f;
  }
}

// ---------------------------------------------------------------- layouts

// A token that counts, for the backward: those that do not are left out of all its products.
struct __align__(16) Token {
  float lse, dloss;
  int32_t target, row;
};

// fp32 x [T][d], n = T d, to its parts [3][T][d]; with a list its tokens' rows alone, one after another.
__global__ __launch_bounds__(kThreads) void head_split_kernel(const float* __restrict__ x, uint16_t* __restrict__ parts,
                                                              size_t n, int d, const Token* __restrict__ list,
                                                              const int* __restrict__ count) {
  const size_t i = (static_cast<size_t>(blockIdx.x) * kThreads + threadIdx.x) * 4;
  if (i >= n) return;
  size_t from = i;
  if (list != nullptr) {
    const uint32_t four = static_cast<uint32_t>(i / 4), t = four / (d / 4);
    if (t >= static_cast<uint32_t>(*count)) return;
    from = static_cast<size_t>(list[t].row) * d + (four - t * (d / 4)) * 4;
  }
  const f32x4 v = *reinterpret_cast<const f32x4*>(x + from);
  uint32_t p[4][3];
#pragma unroll
  for (int j = 0; j < 4; ++j) bf16_parts(v[j], p[j]);
#pragma unroll
  for (int k = 0; k < 3; ++k)
    *reinterpret_cast<u32x2*>(parts + k * n + i) = u32x2{p[0][k] | p[1][k] << 16, p[2][k] | p[3][k] << 16};
}

// The maxima of kMostBlocks fixed ranges, for a wave of each consumer to take the largest of.
constexpr int kMostBlocks = 256;
static_assert(kMostBlocks == 4 * kWave, "four a lane");

__device__ __forceinline__ float wave_most(float m) {
#pragma unroll
  for (int off = kWave / 2; off > 0; off >>= 1) m = fmaxf(m, __shfl_xor(m, off, kWave));
  return m;
}
__device__ __forceinline__ void put_most(float m, float* most) {
  __shared__ float waves[16];
  m = wave_most(m);
  if ((threadIdx.x & (kWave - 1)) == 0) waves[threadIdx.x / kWave] = m;
  __syncthreads();
  if (threadIdx.x != 0) return;
  for (int w = 1; w < static_cast<int>(blockDim.x) / kWave; ++w) m = fmaxf(m, waves[w]);
  most[blockIdx.x] = m;
}

__device__ __forceinline__ bool counts(const int32_t* targets, int t, int vocab) {
  return static_cast<uint32_t>(targets[t]) < static_cast<uint32_t>(vocab);
}

// The list of the tokens that count, in their order, and their number; the largest finite |x| of theirs and (with a dloss)
// the largest |dloss|; zeros to the others' rows of dx.
template <typename T>
__global__ __launch_bounds__(1024) void head_list_kernel(const T* __restrict__ x, const float* __restrict__ lse,
                                                         const float* __restrict__ dloss,
                                                         const int32_t* __restrict__ targets, int tokens, int d, int vocab,
                                                         Token* __restrict__ list, int* __restrict__ count,
                                                         float* __restrict__ most, float* __restrict__ most_x,
                                                         T* __restrict__ dx) {
  constexpr int kWaves = 1024 / kWave;
  __shared__ int earlier[kWaves], here[kWaves];
  const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = tid / kWave;
  for (int64_t first = blockIdx.x * 1024; first < tokens; first += kMostBlocks * 1024) {
    int before = 0;                       // of the tokens ahead of these 1,024, counted by every workgroup for itself
#pragma unroll 8
    for (int t = tid; t < first; t += 1024) before += counts(targets, t, vocab) ? 1 : 0;
#pragma unroll
    for (int off = kWave / 2; off > 0; off >>= 1) before += __shfl_xor(before, off, kWave);
    const int t = static_cast<int>(first) + tid;
    const bool on = t < tokens && counts(targets, t, vocab);
    const uint64_t ballot = __ballot(on);
    if (lane == 0) {
      earlier[wave] = before;
      here[wave] = __popcll(ballot);
    }
    __syncthreads();
    int at = __popcll(ballot & lanemask_lt()), all = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      at += earlier[w] + (w < wave ? here[w] : 0);
      all += earlier[w] + here[w];
    }
    if (on) list[at] = Token{lse[t], dloss ? dloss[t] : 1.f, targets[t], t};
    if (tid == 0 && first + 1024 >= tokens) *count = all;
    __syncthreads();
  }
  typedef T eight __attribute__((ext_vector_type(8), aligned(16)));
  static_assert(alignof(eight) == 16, "what x and dx are aligned to (eight fp32 by themselves claim 32 bytes)");
  const uint32_t row = d / 8, pieces = static_cast<uint32_t>(tokens) * row;       // at most 2^31
  float m = 0.f;
#pragma unroll 4
  for (uint32_t i = blockIdx.x * 1024 + tid; i < pieces; i += kMostBlocks * 1024) {
    const eight v = *reinterpret_cast<const eight*>(x + static_cast<int64_t>(i) * 8);
    if (counts(targets, static_cast<int>(i / row), vocab)) {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float a = fabsf(static_cast<float>(v[j]));
        m = a < INFINITY ? fmaxf(m, a) : m;
      }
    } else {
      *reinterpret_cast<eight*>(dx + static_cast<int64_t>(i) * 8) = eight{};
    }
  }
  put_most(m, most_x);
  if (!dloss) return;
  m = 0.f;
  for (int t = blockIdx.x * 1024 + tid; t < tokens; t += kMostBlocks * 1024)
    if (counts(targets, t, vocab)) m = fmaxf(m, fabsf(dloss[t]));
  __syncthreads();
  put_most(m, most);
}

// The largest of the blocks' maxima, to every lane.
__device__ __forceinline__ float all_most(const float* most) {
  const f32x4 m = reinterpret_cast<const f32x4*>(most)[threadIdx.x & (kWave - 1)];
  return wave_most(fmaxf(fmaxf(m.x, m.y), fmaxf(m.z, m.w)));
}

// The power of two that x is multiplied by: it takes the largest to between 2^14 and 2^15.
__device__ __forceinline__ int x_shift(const float* most) {
  const float m = all_most(most);
  int e = 0;
  frexpf(m, &e);
  return m > 0.f ? 15 - e : 0;
}

// Part i of a value as fp16 parts; what is past the first part of a value that is infinite or none is zero.
__device__ __forceinline__ uint32_t f16_part(float x, int i) {
  const _Float16 hi = static_cast<_Float16>(x);
  if (i == 0) return __builtin_bit_cast(uint16_t, hi);
  const float v = static_cast<float>(hi);
  return fabsf(v) < INFINITY ? __builtin_bit_cast(uint16_t, static_cast<_Float16>(x - v)) : 0u;
}

// in [rows, cols] (cols a multiple of 8) to out [parts][cols][ld] (ld a multiple of 64), zeros from `rows` on, to a multiple of 64.  With
// a list its tokens' rows alone, one after another, and bf16 ones to `copy` as they are.  With `most` as fp16 parts of the
// shifted values; without as the bits they are.  Every load is under way before the first is waited for: of 1,032 x 1,032
// fp32 to two parts 13.8 us with a load at a time, so 5.3.
template <typename T, int PARTS>
__global__ __launch_bounds__(kThreads) void head_transpose_kernel(const T* __restrict__ in, int rows, int cols,
                                                                  uint16_t* __restrict__ out, int64_t ld,
                                                                  const float* __restrict__ most,
                                                                  const Token* __restrict__ list,
                                                                  const int* __restrict__ count,
                                                                  T* __restrict__ copy) {
  constexpr int kN = 16 / sizeof(T), kAcross = 64 / kN, kPieces = 64 * kAcross / kThreads;
  typedef T piece __attribute__((ext_vector_type(kN)));
  __shared__ uint16_t tile[PARTS][64][66];
  const int r0 = blockIdx.x * 64, c0 = blockIdx.y * 64;
  const int in_c = (threadIdx.x % kAcross) * kN, in_r = threadIdx.x / kAcross;
  const int c = min(c0 + in_c, cols - kN);
  if (list != nullptr) {
    rows = *count;
    if (r0 >= rows) return;
  }
  piece v[kPieces];
#pragma unroll
  for (int i = 0; i < kPieces; ++i) {
    const int r = min(r0 + in_r + i * (kThreads / kAcross), rows - 1);
    v[i] = *reinterpret_cast<const piece*>(in + static_cast<int64_t>(list ? list[r].row : r) * cols + c);
  }
  const int shift = most ? x_shift(most) : 0;
#pragma unroll
  for (int i = 0; i < kPieces; ++i) {
    const int at = in_r + i * (kThreads / kAcross);
    const bool on = r0 + at < rows;
    if (copy != nullptr && on && c0 + in_c < cols)
      *reinterpret_cast<piece*>(copy + static_cast<int64_t>(r0 + at) * cols + c) = v[i];
#pragma unroll
    for (int j = 0; j < kN; ++j) {
      uint32_t p[PARTS] = {};
      if (most) {
        float x;
        if constexpr (sizeof(T) == 4) x = ldexpf(v[i][j], shift);
        else x = ldexpf(bits_f32(v[i][j]), shift);
#pragma unroll
        for (int k = 0; k < PARTS; ++k) p[k] = f16_part(x, k);
      } else if constexpr (sizeof(T) == 2) {
        p[0] = v[i][j];
      }
#pragma unroll
      for (int k = 0; k < PARTS; ++k) tile[k][in_c + j][at] = static_cast<uint16_t>(on ? p[k] : 0u);
    }
  }
  __syncthreads();
  const int64_t part = static_cast<int64_t>(cols) * ld;
#pragma unroll
  for (int k = 0; k < PARTS; ++k)
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int row = i * 32 + threadIdx.x / 8, at = (threadIdx.x % 8) * 8;
      const uint32_t* from = reinterpret_cast<const uint32_t*>(&tile[k][row][at]);
      if (c0 + row < cols)
        *reinterpret_cast<u32x4*>(out + k * part + static_cast<int64_t>(c0 + row) * ld + r0 + at) =
            u32x4{from[0], from[1], from[2], from[3]};
    }
}

// ---------------------------------------------------------------- forward

// Each token's (reference, sum of exp(z - reference)) over the tile's rows of W, to stats[tile][T], in units of u, the
// product with its sign turned where scale is below 0: z = |scale| u (and spread_of).  The reference is the largest u, or 0
// where that is infinite or none; with a sum of 0 it is -infinity, so that it raises no other's.  goal[t]: the target's u,
// by the tile that holds it.  The end of a tile takes 8 clocks of a lane's for each logit, 4 of them exp2's: with the target
// and W's last row looked for at each the kernel took 1.05 times as long.
constexpr float kLog2e = 1.44269504f;
// What the products are multiplied by, so that |scale| log2(e) does not overflow; scale / it takes scale's place.
__host__ __device__ __forceinline__ float spread_of(float scale) { return fabsf(scale) > 1e38f ? 4.f : 1.f; }

template <int BM, int BN, int WR, int WC, int GROUPS, TileParts PARTS>
__global__ __launch_bounds__(64 * WR * WC * GROUPS) void head_stats_kernel(TilePairs p, int tiles_m, int tiles_n, float scale,
                                                                          const int32_t* __restrict__ targets,
                                                                          float2* __restrict__ stats,
                                                                          float* __restrict__ goal) {
  typedef Tile<false, BM, BN, WR, WC, 2, PARTS, GROUPS> Tl;
  constexpr int MT = Tl::MT, NT = Tl::NE;
  __shared__ __align__(16) uint16_t buf0[GROUPS * Tl::kElems];
  __shared__ __align__(16) uint16_t buf1[GROUPS * Tl::kElems];
  __shared__ float2 waves[WR][BN];
  const int item = tile_item(tiles_m * tiles_n);
  if (item >= tiles_m * tiles_n) return;                    // the whole workgroup: no barrier is skipped
  const TilePlace at = tile_place(item, tiles_m, tiles_n);
  Tl tile;
  tile.init(p, at.m * BM, at.n * BN);
  const int group = Tl::group(), own = group * Tl::kElems;
  f32x4 all[MT][Tl::NT], acc[MT][NT];
  tile.run(p, 0, Tl::slices(p), buf0 + own, buf1 + own, nullptr, nullptr, all);
  Tl::share(all, buf0, acc);
  const int lane = threadIdx.x & 63, wave = Tl::thread() >> 6, wr = wave / WC, wc = wave % WC;
  const int V = p.a_rows, T = p.b_rows;
  const int v0 = at.m * BM + wr * MT * 16 + 4 * (lane >> 4);
  const float spread = spread_of(scale), turn = scale < 0.f ? -spread : spread, c = fabsf(scale) / spread * kLog2e;
  const bool edge = at.m * BM + BM > V;                     // (uniform: W's last rows)
#pragma unroll
  for (int j = 0; j < NT; ++j) {
    const int n = (wc * Tl::NT + group * NT + j) * 16 + (lane & 15), t = at.n * BN + n;
    if (turn != 1.f) {
#pragma unroll
      for (int i = 0; i < MT; ++i) acc[i][j] *= turn;
    }
    const int in = (t < T ? targets[t] : -1) - v0;          // the target's entry, which few waves hold one of
    const bool holds = in >= 0 && in < MT * 16 && (in & 15) < 4 && v0 + in < V;
    if (__any(holds)) {
#pragma unroll
      for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if (holds && in == 16 * i + r) goal[t] = acc[i][j][r];
    }
    float top = -INFINITY, sum = 0.f;
    const auto over = [&](auto last) {
      const auto there = [&](int i, int r) { return !last || v0 + i * 16 + r < V; };
#pragma unroll
      for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r) top = there(i, r) ? fmaxf(top, acc[i][j][r]) : top;
      top = fmaxf(top, __shfl_xor(top, 16, 64));
      top = fmaxf(top, __shfl_xor(top, 32, 64));
      top = fabsf(top) < INFINITY ? top : 0.f;
#pragma unroll
      for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r) sum += there(i, r) ? __builtin_amdgcn_exp2f((acc[i][j][r] - top) * c) : 0.f;
    };
    if (edge) over(std::true_type());
    else over(std::false_type());
    sum += __shfl_xor(sum, 16, 64);
    sum += __shfl_xor(sum, 32, 64);
    if (lane < 16) waves[wr][n] = float2{sum == 0.f ? -INFINITY : top, sum};
  }
  __syncthreads();
  for (int n = threadIdx.x; n < BN; n += Tl::kThreads * GROUPS) {
    const int t = at.n * BN + n;
    if (t >= T) continue;
    float top = waves[0][n].x;
#pragma unroll
    for (int w = 1; w < WR; ++w) top = fmaxf(top, waves[w][n].x);
    float sum = 0.f;
#pragma unroll
    for (int w = 0; w < WR; ++w)
      if (waves[w][n].y != 0.f) sum += waves[w][n].y * __builtin_amdgcn_exp2f((waves[w][n].x - top) * c);
    stats[static_cast<int64_t>(at.m) * T + t] = float2{top, sum};
  }
}

// The tiles' pairs of each token, 16 lanes a token, added in fp64 in the order of the tiles; scale here is u's factor.
__global__ __launch_bounds__(kThreads) void head_join_kernel(const float2* __restrict__ stats,
                                                             const float* __restrict__ goal,
                                                             const int32_t* __restrict__ targets, int T, int vocab,
                                                             int tiles, double scale, float* __restrict__ loss,
                                                             float* __restrict__ lse) {
  __shared__ float tops[16][17];
  __shared__ double sums[16][17];
  const int n = threadIdx.x % 16, q = threadIdx.x / 16, t = blockIdx.x * 16 + n;
  float top = -INFINITY;
  if (t < T)
    for (int i = q; i < tiles; i += 16) top = fmaxf(top, stats[static_cast<int64_t>(i) * T + t].x);
  tops[q][n] = top;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 16; ++i) top = fmaxf(top, tops[i][n]);
  double sum = 0.0;
  if (t < T)
    for (int i = q; i < tiles; i += 16) {
      const float2 s = stats[static_cast<int64_t>(i) * T + t];
      if (s.y != 0.f) sum += s.y * exp((static_cast<double>(s.x) - top) * scale);
    }
  sums[q][n] = sum;
  __syncthreads();
  if (q != 0 || t >= T) return;
  sum = 0.0;
#pragma unroll
  for (int i = 0; i < 16; ++i) sum += sums[i][n];
  const double all = top * scale + log(sum);
  lse[t] = static_cast<float>(all);
  loss[t] = counts(targets, t, vocab) ? static_cast<float>(all - goal[t] * scale) : 0.f;
}

// The same with a workgroup a token, for few tokens.
__global__ __launch_bounds__(kThreads) void head_join_few_kernel(const float2* __restrict__ stats,
                                                                 const float* __restrict__ goal,
                                                                 const int32_t* __restrict__ targets, int T, int vocab,
                                                                 int tiles, double scale, float* __restrict__ loss,
                                                                 float* __restrict__ lse) {
  __shared__ float tops[kThreads / kWave];
  __shared__ double sums[kThreads / kWave];
  const int t = blockIdx.x, wave = threadIdx.x / kWave;
  constexpr int kHeld = 8;                                  // pairs a thread holds while the maximum is found
  float2 held[kHeld];
  float top = -INFINITY;
#pragma unroll
  for (int j = 0; j < kHeld; ++j) {
    const int i = threadIdx.x + j * kThreads;
    held[j] = i < tiles ? stats[static_cast<int64_t>(i) * T + t] : float2{-INFINITY, 0.f};
    top = fmaxf(top, held[j].x);
  }
  for (int i = threadIdx.x + kHeld * kThreads; i < tiles; i += kThreads)
    top = fmaxf(top, stats[static_cast<int64_t>(i) * T + t].x);
  top = wave_most(top);
  if ((threadIdx.x & (kWave - 1)) == 0) tops[wave] = top;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kThreads / kWave; ++w) top = fmaxf(top, tops[w]);
  double sum = 0.0;
#pragma unroll
  for (int j = 0; j < kHeld; ++j)
    if (held[j].y != 0.f) sum += held[j].y * exp((static_cast<double>(held[j].x) - top) * scale);
  for (int i = threadIdx.x + kHeld * kThreads; i < tiles; i += kThreads) {
    const float2 s = stats[static_cast<int64_t>(i) * T + t];
    if (s.y != 0.f) sum += s.y * exp((static_cast<double>(s.x) - top) * scale);
  }
#pragma unroll
  for (int off = kWave / 2; off > 0; off >>= 1) sum += __shfl_xor(sum, off, kWave);
  if ((threadIdx.x & (kWave - 1)) == 0) sums[wave] = sum;
  __syncthreads();
  if (threadIdx.x != 0) return;
#pragma unroll
  for (int w = 1; w < kThreads / kWave; ++w) sum += sums[w];
  const double all = top * scale + log(sum);
  lse[t] = static_cast<float>(all);
  loss[t] = counts(targets, t, vocab) ? static_cast<float>(all - goal[t] * scale) : 0.f;
}

// ---------------------------------------------------------------- backward

// The largest |dloss|; 1 without any, or where it is no finite number above 0.
__device__ __forceinline__ float most_of(const float* most) {
  if (most == nullptr) return 1.f;
  const float m = all_most(most);
  return m > 0.f && m < INFINITY ? m : 1.f;
}

// r of a piece of the vocabulary, over s and the largest dloss: rows[part][T][piece] in PR bf16 parts, and times 2^15
// cols[part][piece][t_ld] in PC fp16 parts; zeros past the piece's rows of W and past the tokens.
// lost: what of a target's r one bf16 part of it does not hold, [T] (of it alone r is near the largest dloss in most
// tokens; dx adds it times W's row: half the error of dx is without that from there).
// The tile's rows are in an order in which a lane holds 8 values of W's rows one after another, and NT tokens one after another, so
// that both orders are written from the registers, in whole 64- and 128-byte pieces.  (Through LDS, a part at a time,
// the end of a tile took as long as its products: 7,168 x 8,192 of 2,048 316 us, so 258, 0.93 PFLOP/s.)
constexpr int kSlopeBits = 15;
constexpr float kSlopeUp = 1 << kSlopeBits;

// Within a wave's rows of A, accumulator block i, row 4 q + r (q = lane / 16): 32 (i / 2) + 8 q + 4 (i % 2) + r; within its
// rows of B, block j, row l: NT l + j.
struct SlopeRowA {
  __device__ __forceinline__ int operator()(int row) const {
    const int i = (row >> 4) & 1, q = (row >> 2) & 3;
    return (row & ~31) | q << 3 | i << 2 | (row & 3);
  }
};
template <int NT>
struct SlopeRowB {
  __device__ __forceinline__ int operator()(int row) const {
    const int in = row % (16 * NT);
    return row - in + (in & 15) * NT + (in >> 4);
  }
};

template <int BM, int BN, int WR, int WC, int GROUPS, TileParts PARTS, int PR, int PC>
__global__ __launch_bounds__(64 * WR * WC * GROUPS) void head_slope_kernel(TilePairs p, int tiles_m, int of, float scale,
                                                                 const Token* __restrict__ list,
                                                                 const int* __restrict__ count,
                                                                 const float* __restrict__ most, int v_first,
                                                                 int piece, int t_ld, uint16_t* __restrict__ rows,
                                                                 uint16_t* __restrict__ cols,
                                                                 float* __restrict__ lost) {
  typedef Tile<false, BM, BN, WR, WC, 2, PARTS, GROUPS> Tl;
  constexpr int MT = Tl::MT, NT = Tl::NE;
  static_assert(MT % 2 == 0 && (NT == 1 || NT == 2 || NT == 4), "pieces of 16 bytes along W's rows, of NT along the tokens");
  __shared__ __align__(16) uint16_t buf0[GROUPS * Tl::kElems];
  __shared__ __align__(16) uint16_t buf1[GROUPS * Tl::kElems];
  const int T = *count, tiles_n = (T + BN - 1) / BN;
  p.b_rows = T;
  const int item = tile_item(tiles_m * tiles_n);
  if (item >= tiles_m * tiles_n) return;
  const TilePlace at = tile_place<8>(item, tiles_m, tiles_n);        // (bands of 8: 258 us, of 4 272)
  Tl tile;
  tile.init(p, at.m * BM, at.n * BN, SlopeRowA(), SlopeRowB<Tl::NT>());
  const int group = Tl::group(), own = group * Tl::kElems;
  f32x4 all[MT][Tl::NT], acc[MT][NT];
  tile.run(p, 0, Tl::slices(p), buf0 + own, buf1 + own, nullptr, nullptr, all);
  Tl::share(all, buf0, acc);
  const int lane = threadIdx.x & 63, wave = Tl::thread() >> 6, wr = wave / WC, wc = wave % WC;
  const int V = p.a_rows;
  const int v0 = at.m * BM + wr * MT * 16 + 8 * (lane >> 4);       // acc[i][j][r]: row v0 + 32 (i / 2) + 4 (i % 2) + r
  const int t0 = at.n * BN + wc * Tl::NT * 16 + Tl::NT * (lane & 15) + group * NT;     // token t0 + j
  const float largest = most_of(most);
#pragma unroll
  for (int j = 0; j < NT; ++j) {
    const int t = t0 + j;
    const bool on = t < T;
    const Token token = list[min(t, T - 1)];
    const int y = token.target;
    const float l = token.lse, g = token.dloss / largest;
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
      for (int r = 0; r < 4; ++r) acc[i][j][r] = __expf(fmaf(acc[i][j][r], scale, -l));
    // the target's entry, which few waves hold one of
    const int in = y - v_first - v0;
    const bool holds = on && in >= 0 && in < MT * 16 && (in & 31) < 8;
    const int which = (in >> 5) * 8 + (in & 7);
    if (__any(holds)) {
#pragma unroll
      for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if (holds && which == 4 * i + r) {
            acc[i][j][r] -= 1.f;
            if (PR == 1) {
              const float whole = g * acc[i][j][r], part = bits_f32(bf16_bits(whole));
              lost[t] = fabsf(part) <= 3.4e38f ? whole - part : 0.f;
            }
          }
    }
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
      for (int r = 0; r < 4; ++r) acc[i][j][r] = on ? g * acc[i][j][r] : 0.f;
  }
  if (at.m * BM + BM > V) {               // (uniform: the last rows of W)
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
      for (int r = 0; r < 4; ++r)
        if (v0 + 32 * (i / 2) + 4 * (i % 2) + r >= V) {
#pragma unroll
          for (int j = 0; j < NT; ++j) acc[i][j][r] = 0.f;
        }
  }
  // (piece is a multiple of BM)
  const int64_t by_row = static_cast<int64_t>(of) * piece, by_col = static_cast<int64_t>(piece) * t_ld;
#pragma unroll
  for (int j = 0; j < NT; ++j) {
    if (t0 + j >= T) continue;
    uint16_t* to = rows + static_cast<int64_t>(t0 + j) * piece + v0;
#pragma unroll
    for (int i = 0; i < MT; i += 2) {
      uint32_t b[8][PR];
#pragma unroll
      for (int e = 0; e < 8; ++e) bf16_parts(acc[i + e / 4][j][e % 4], b[e]);
#pragma unroll
      for (int k = 0; k < PR; ++k)
        *reinterpret_cast<u32x4*>(to + k * by_row + 16 * i) =
            u32x4{b[0][k] | b[1][k] << 16, b[2][k] | b[3][k] << 16, b[4][k] | b[5][k] << 16, b[6][k] | b[7][k] << 16};
    }
  }
  if (t0 >= t_ld) return;
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      uint16_t* to = cols + static_cast<int64_t>(v0 + 32 * (i / 2) + 4 * (i % 2) + r) * t_ld + t0;
#pragma unroll
      for (int k = 0; k < PC; ++k) {
        uint32_t b[NT];
#pragma unroll
        for (int j = 0; j < NT; ++j) b[j] = f16_part(acc[i][j][r] * kSlopeUp, k);
        if constexpr (NT == 4) *reinterpret_cast<u32x2*>(to + k * by_col) = u32x2{b[0] | b[1] << 16, b[2] | b[3] << 16};
        else if constexpr (NT == 2) *reinterpret_cast<uint32_t*>(to + k * by_col) = b[0] | b[1] << 16;
        else to[k * by_col] = static_cast<uint16_t>(b[0]);
      }
    }
}

// A product whose m lies along the rows of the output, [n][m] of ld.  Of one split of k: out = (D + before) f (dx) or
// D f + before (dW: whole = false), each without `before` where it is not given, f = scale times the largest dloss, and of
// shifted operands (x_most) what takes their shifts back.  Of
// several, split i's D is added to sums[i], or written there where first is set.
struct ProductArgs {
  int tiles_m, tiles_n, splits;
  float *sums, *before;
  bool first, whole;
  void* out;
  int64_t ld;
  float scale;
  const float *most, *x_most;
  const int* count;       // tokens that count: rows n, or (along_k) k of the product
  bool along_k;
  const Token* list;      // given where row n goes to its token's place in out
  const float* lost;      // [n], times W's row of the target is added to D
  const uint16_t* w;
  int64_t sum_size;       // from one split's sums to the next's
};

// What is added to row t of dx, columns m .. m + 3, before it is scaled.
__device__ __forceinline__ f32x4 lost_row(const ProductArgs& g, int t, int m) {
  const u32x2 b = *reinterpret_cast<const u32x2*>(g.w + g.list[t].target * g.ld + m);
  return g.lost[t] * f32x4{bits_f32(b.x & 0xffffu), bits_f32(b.x >> 16), bits_f32(b.y & 0xffffu), bits_f32(b.y >> 16)};
}

// What the sums are multiplied by, 2^e m with m below 1, as neither its own parts nor a sum times one of them need be within
// fp32 where the result is.
struct Factor {
  float m;
  int e;
  __device__ __forceinline__ float operator()(float v) const { return ldexpf(v * m, e); }
};
__device__ __forceinline__ Factor product_factor(const ProductArgs& g) {
  int e = 0;
  const double m = frexp(static_cast<double>(g.scale) * most_of(g.most), &e);
  return {static_cast<float>(m), g.x_most ? e - kSlopeBits - x_shift(g.x_most) : e};
}

// GROUPS sets of waves share a tile's slices where there are too few tiles for more than one on a CU: with one wave on each
// of its parts a CU waits for every slice.
template <bool F16, typename OT, int BM, int BN, int WR, int WC, int GROUPS, TileParts PARTS>
__global__ __launch_bounds__(64 * WR * WC * GROUPS) void head_product_kernel(TilePairs p, ProductArgs g) {
  typedef Tile<F16, BM, BN, WR, WC, 2, PARTS, GROUPS> Tl;
  __shared__ __align__(16) uint16_t buf0[GROUPS * Tl::kElems];
  __shared__ __align__(16) uint16_t buf1[GROUPS * Tl::kElems];
  const int counted = *g.count;
  if (g.along_k) {
    p.k = (counted + 63) / 64 * 64;
  } else {
    p.b_rows = counted;
    g.tiles_n = (counted + BN - 1) / BN;
  }
  const int tiles = g.tiles_m * g.tiles_n, id = tile_item(tiles * g.splits);
  if (id >= tiles * g.splits) return;
  const int split = id / tiles;
  const TilePlace at = tile_place(id - split * tiles, g.tiles_m, g.tiles_n);
  Tl tile;
  tile.init(p, at.m * BM, at.n * BN);
  f32x4 acc[Tl::MT][Tl::NT];
  const int64_t slices = Tl::slices(p);
  const int group = Tl::group(), own = group * Tl::kElems;
  const int from = static_cast<int>(slices * split / g.splits), to = static_cast<int>(slices * (split + 1) / g.splits);
  if (to > from) {
    tile.run(p, from, to, buf0 + own, buf1 + own, nullptr, nullptr, acc);
  } else {                                // (no token counts)
#pragma unroll
    for (int i = 0; i < Tl::MT; ++i)
#pragma unroll
      for (int j = 0; j < Tl::NT; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  if constexpr (GROUPS > 1) {             // the first group adds what the others have, in their order, and goes on alone
    static_assert((GROUPS - 1) * BM * BN * 4 <= GROUPS * Tl::kElems * 2, "the groups' sums fit a buffer");
    f32x4* sums = reinterpret_cast<f32x4*>(buf0) + Tl::thread();
    __syncthreads();
#pragma unroll
    for (int j = 0; j < Tl::NT; ++j)
#pragma unroll
      for (int i = 0; i < Tl::MT; ++i)
        if (group > 0) sums[((group - 1) * Tl::MT * Tl::NT + j * Tl::MT + i) * Tl::kThreads] = acc[i][j];
    __syncthreads();
    if (group > 0) return;
#pragma unroll
    for (int k = 0; k < GROUPS - 1; ++k)
#pragma unroll
      for (int j = 0; j < Tl::NT; ++j)
#pragma unroll
        for (int i = 0; i < Tl::MT; ++i) acc[i][j] += sums[(k * Tl::MT * Tl::NT + j * Tl::MT + i) * Tl::kThreads];
  }
  const int lane = threadIdx.x & 63, wave = Tl::thread() >> 6, wr = wave / WC, wc = wave % WC;
  const Factor f = product_factor(g);
#pragma unroll
  for (int j = 0; j < Tl::NT; ++j) {
    const int n = at.n * BN + (wc * Tl::NT + j) * 16 + (lane & 15);
    if (n >= p.b_rows) continue;
    const int64_t out_row = g.list ? g.list[n].row : n;
#pragma unroll
    for (int i = 0; i < Tl::MT; ++i) {
      const int m = at.m * BM + (wr * Tl::MT + i) * 16 + 4 * (lane >> 4);
      if (m >= p.a_rows) continue;
      const int64_t o = n * g.ld + m;
      f32x4 v = acc[i][j];
      if (g.splits > 1) {
        float* sum = g.sums + split * g.sum_size + o;
        if (!g.first) v += *reinterpret_cast<const f32x4*>(sum);
        *reinterpret_cast<f32x4*>(sum) = v;
        continue;
      }
      if (g.whole && g.before) v += *reinterpret_cast<const f32x4*>(g.before + o);
      if (g.lost) v += lost_row(g, n, m);
#pragma unroll
      for (int r = 0; r < 4; ++r) v[r] = f(v[r]);
      if (!g.whole && g.before) v += *reinterpret_cast<const f32x4*>(g.before + o);
      OT* out = static_cast<OT*>(g.out) + out_row * g.ld + m;
      if constexpr (sizeof(OT) == 4)
        *reinterpret_cast<f32x4*>(out) = v;
      else
        *reinterpret_cast<u32x2*>(out) =
            u32x2{bf16_bits(v.x) | bf16_bits(v.y) << 16, bf16_bits(v.z) | bf16_bits(v.w) << 16};
    }
  }
}

// dx from the splits' sums, in their order.
template <typename OT>
__global__ __launch_bounds__(kThreads) void head_sum_kernel(ProductArgs g, int rows) {
  const Factor f = product_factor(g);
  const int64_t i = (static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x) * 4;
  if (i >= (g.along_k ? rows : *g.count) * g.ld) return;
  f32x4 v = *reinterpret_cast<const f32x4*>(g.sums + i);
  for (int s = 1; s < g.splits; ++s) v += *reinterpret_cast<const f32x4*>(g.sums + s * g.sum_size + i);
  const int t = static_cast<int>(i / g.ld), m = static_cast<int>(i - t * g.ld);
  if (g.lost) v += lost_row(g, t, m);
#pragma unroll
  for (int r = 0; r < 4; ++r) v[r] = f(v[r]);
  if (!g.whole && g.before) v += *reinterpret_cast<const f32x4*>(g.before + i);
  OT* out = static_cast<OT*>(g.out) + (g.list ? g.list[t].row * g.ld + m : i);
  if constexpr (sizeof(OT) == 4)
    *reinterpret_cast<f32x4*>(out) = v;
  else
    *reinterpret_cast<u32x2*>(out) = u32x2{bf16_bits(v.x) | bf16_bits(v.y) << 16, bf16_bits(v.z) | bf16_bits(v.w) << 16};
}

// ---------------------------------------------------------------- host

size_t up256(size_t x) { return (x + 255) & ~static_cast<size_t>(255); }
int64_t up(int64_t x, int64_t to) { return (x + to - 1) / to * to; }

// A product's tiles, and how often its slices are split, by what the sizes of tile measured (us a slice): 256 x 256,
// eight waves and a CU to itself, 1.7; 128 x 128, two to a CU, 0.95 both, 0.7 alone; 64 x 64, up to four to a CU, 0.25 alone
// and 0.2 more with each beside it.  So large tiles where there is one for each CU (7,168 x 8,192 over 2,048: 1.7 a slice
// for 16 tiles of 64 x 64, which take 3.4), small ones where there are few: 600 x 2,314 over 1,696 46 in 27 large ones, 20 in
// 95 of 128 x 128.  Small ones are taken up to 4,096 of them.
constexpr int kCus = 256, kManyTiles = 4096;
struct TilePlan {
  int side, splits;
};
TilePlan tile_plan(int64_t m, int64_t n, int slices, int most_splits, bool largest) {
  TilePlan best{64, 1};
  double least = 1e300;
  for (int side : {64, 128, 256}) {
    const int64_t tiles = ((m + side - 1) / side) * ((n + side - 1) / side);
    if (side == 256 ? !largest : tiles > (side == 128 && !largest ? INT64_MAX : kManyTiles)) continue;
    for (int s = 1; s <= most_splits && (s == 1 || 8 * s <= slices); ++s) {
      const int64_t full = (tiles * s + kCus - 1) / kCus;   // of the fullest CU
      const double each = (slices + s - 1) / s, whole = static_cast<double>(full);
      double us = s > 1 ? 4.0 + 8e-6 * m * n * s / 3.0 : 0.0;
      if (side == 256) us += whole * (4.0 + 1.7 * each);
      else if (side == 128) us += static_cast<double>(full / 2) * (4.0 + 0.95 * each) + (full % 2 ? 4.0 + 0.7 * each : 0.0);
      else us += static_cast<double>(full / 4) * (4.0 + 0.85 * each) + (full % 4 ? 3.0 + (0.05 + 0.2 * (full % 4)) * each : 0.0);
      if (us < least) {
        least = us;
        best = {side, s};
      }
    }
  }
  return best;
}
int slice_count(int64_t k, int pairs) { return static_cast<int>((k + kTileBK - 1) / kTileBK) * pairs; }

int x_parts(const umem_head_desc& hd) { return hd.xtype == UMEM_F32 ? 3 : 1; }
int row_parts(const umem_head_desc& hd) { return hd.xtype == UMEM_F32 ? 3 : 1; }       // of r, for dx
int col_parts(const umem_head_desc& hd) { return hd.gtype == UMEM_F32 ? 2 : 1; }       // of r, for dW
int x_col_parts(const umem_head_desc& hd) { return hd.xtype == UMEM_F32 && hd.gtype == UMEM_F32 ? 2 : 1; }

// Rows of the vocabulary in a piece of the backward.  r's scratch holds 2^26 values of a part in each order at most (from
// 2^18 tokens on 256 rows of every token), W's transposed piece 2^14 rows.
constexpr int64_t kPieceRows = 1 << 14, kPieceValues = 1 << 26;
int64_t most_piece(const umem_head_desc& hd) { return std::min(kPieceRows, up(hd.vocab, 256)); }
// Elements of a row that holds all tokens: T in whole slices, and a line more, as rows a large power of two apart
// are written and read slower.
int64_t token_row(int T) { return up(T, 64) + 64; }
int64_t piece_values(const umem_head_desc& hd, int T) {
  const int64_t t = token_row(T);
  return std::min(t * most_piece(hd), std::max(kPieceValues, t * 256));
}
int piece_rows(const umem_head_desc& hd, int T) {
  const int64_t t = token_row(T), most = std::min(most_piece(hd), std::max<int64_t>(256, piece_values(hd, T) / t / 256 * 256));
  const int64_t pieces = (hd.vocab + most - 1) / most;
  return static_cast<int>(up((hd.vocab + pieces - 1) / pieces, 256));
}

// The products of the gradients: k is split where tiles are few.  (Tiles that are split are as many, with their splits, as the
// chip holds at most: four of 64 x 64 a CU, two of 128 x 128, one of 256 x 256.)
constexpr int kMostSplits = 32;
constexpr size_t kSumValues = static_cast<size_t>(kCus) * 256 * 256;
TilePlan split_plan(int64_t m, int64_t n, int slices) {
  TilePlan p = tile_plan(m, n, slices, kMostSplits, true);
  const int64_t tiles = (up(m, p.side) / p.side) * (up(n, p.side) / p.side);
  const int64_t most = p.side == 256 ? kCus : p.side == 128 ? 2 * kCus : 4 * kCus;
  p.splits = static_cast<int>(std::max<int64_t>(1, std::min<int64_t>(p.splits, most / tiles)));
  return p;
}
TilePlan dx_plan(const umem_head_desc& hd, int T) {
  return split_plan(hd.d, T, slice_count(piece_rows(hd, T), row_parts(hd)));
}
// (of `rows` rows of the vocabulary: 4,266 tokens by 1,693 of 264 in fp32 57 us in one piece)
TilePlan dw_plan(const umem_head_desc& hd, int T, int rows) {
  const int pairs = col_parts(hd) * x_col_parts(hd) - (col_parts(hd) * x_col_parts(hd) == 4 ? 1 : 0);
  return split_plan(hd.d, rows, slice_count(up(T, 64), pairs));
}
size_t sum_values(const umem_head_desc& hd, int T) {
  const size_t x = static_cast<size_t>(T) * hd.d;
  return std::max(x, std::min(kMostSplits * x, kSumValues));
}

// The forward goes by bands of tokens, so that its scratch and its grids are bounded; a workspace for T tokens holds what
// fewer need.
constexpr int kBandTokens = 1 << 15, kFewTokens = 512;
struct ForwardLayout {
  size_t parts, stats, goal, total;
  ForwardLayout(const umem_head_desc& hd, int T) {
    const size_t t = std::min(T, kBandTokens), d = hd.d, small = (hd.vocab + 63) / 64, large = (hd.vocab + 255) / 256;
    // (4,096 tiles of 64 or 128 tokens' width at most hold 2^19 pairs)
    parts = 0;
    stats = up256(hd.xtype == UMEM_F32 ? 3 * t * d * 2 : 0);
    goal = stats + up256(sizeof(float2) * std::max(large * t, std::min(small * t, size_t{1} << 19)));
    total = goal + up256(t * sizeof(float));
  }
};
struct BackwardLayout {
  size_t parts, xt, wt, rows, cols, sum, sum_w, most, x_most, lost, list, count, total;
  BackwardLayout(const umem_head_desc& hd, int T) {
    const size_t t = T, tp = token_row(T), d = hd.d, values = piece_values(hd, T);
    parts = 0;
    xt = up256((hd.xtype == UMEM_F32 ? 3 : 1) * t * d * 2);
    wt = xt + up256(x_col_parts(hd) * d * tp * 2);
    rows = wt + up256(d * most_piece(hd) * 2);
    cols = rows + up256(row_parts(hd) * values * 2);
    sum = cols + up256(col_parts(hd) * values * 2);
    sum_w = sum + up256(sum_values(hd, T) * sizeof(float));
    most = sum_w + up256(std::min(kMostSplits * d * most_piece(hd), kSumValues) * sizeof(float));
    x_most = most + up256(kMostBlocks * sizeof(float));
    lost = x_most + up256(kMostBlocks * sizeof(float));
    list = lost + up256(t * sizeof(float));
    count = list + up256(t * sizeof(Token));
    total = count + 256;
  }
};

// The logits' operands: rows of W along m, tokens along n.
TilePairs logit_pairs(const umem_head_desc& hd, int T, const void* x, const uint16_t* parts, const uint16_t* w, int v) {
  TilePairs p{};
  p.n = x_parts(hd);
  for (int i = 0; i < p.n; ++i) {
    p.a[i] = w;
    p.b[i] = hd.xtype == UMEM_F32 ? parts + static_cast<size_t>(p.n - 1 - i) * T * hd.d : static_cast<const uint16_t*>(x);
  }
  p.a_rows = v;
  p.b_rows = T;
  p.k = hd.d;
  p.a_ld = p.b_ld = hd.d;
  return p;
}

void split_x(const umem_head_desc& hd, int T, const void* x, uint16_t* parts, const Token* list, const int* count,
             hipStream_t s) {
  const size_t n = static_cast<size_t>(T) * hd.d;
  hipLaunchKernelGGL(head_split_kernel, dim3(static_cast<unsigned>((n / 4 + kThreads - 1) / kThreads)), dim3(kThreads), 0, s,
                     static_cast<const float*>(x), parts, n, hd.d, list, count);
}

template <bool F16, typename OT>
void product(const TilePairs& p, ProductArgs g, int side, hipStream_t s) {
#define UMEM_PRODUCT(BM, WC, GROUPS, PARTS)                                                                     \
  hipLaunchKernelGGL((head_product_kernel<F16, OT, BM, BM, 2, WC, GROUPS, PARTS>), dim3(tile_grid(items)),      \
                     dim3(128 * WC * GROUPS), 0, s, p, g)
  g.tiles_m = (p.a_rows + side - 1) / side;
  g.tiles_n = (p.b_rows + side - 1) / side;
  const int items = g.tiles_m * g.tiles_n * g.splits;
  constexpr TileParts kParts = !F16 && sizeof(OT) == 4 ? kThree : kPlain;       // (dx of fp32 alone has three of r)
  if (side == 256) UMEM_PRODUCT(256, 4, 1, kPlain);
  else if (side == 128 && items > kCus) UMEM_PRODUCT(128, 2, 1, kPlain);
  else if (side == 128) UMEM_PRODUCT(128, 2, 2, kPlain);
  else if (!F16 && p.n == 3 && items > kCus) UMEM_PRODUCT(64, 2, 1, kParts);
  else if (!F16 && p.n == 3) UMEM_PRODUCT(64, 2, 2, kParts);
  else if (items > 2 * kCus) UMEM_PRODUCT(64, 2, 1, kPlain);
  else if (items > kCus) UMEM_PRODUCT(64, 2, 2, kPlain);
  else UMEM_PRODUCT(64, 2, 4, kPlain);
#undef UMEM_PRODUCT
}

template <typename OT>
void sum_splits(const ProductArgs& g, int rows, hipStream_t s) {
  const dim3 grid(static_cast<unsigned>((rows * g.ld / 4 + kThreads - 1) / kThreads));
  hipLaunchKernelGGL(head_sum_kernel<OT>, grid, dim3(kThreads), 0, s, g, rows);
}

template <int PR, int PC>
void slope(const TilePairs& p, float scale, const Token* list, const int* count, const float* most, int v_first, int piece,
           int t_ld, uint16_t* rows, uint16_t* cols, float* lost, hipStream_t s) {
  // (of 256 x 256 tiles one at a time is on a CU, and nothing beside its end)
  const int side = tile_plan(piece, p.b_rows, slice_count(p.k, p.n), 1, false).side;
  const int tm = (piece + side - 1) / side, tn = (p.b_rows + side - 1) / side;
  constexpr TileParts kParts = PR == 3 ? kThree : kPlain;
#define UMEM_SLOPE(BM, GROUPS, PARTS)                                                                            \
  hipLaunchKernelGGL((head_slope_kernel<BM, BM, 2, 2, GROUPS, PARTS, PR, PC>), dim3(tile_grid(tm * tn)),        \
                     dim3(256 * GROUPS), 0, s, p, tm, p.b_rows, scale, list, count, most, v_first, piece, t_ld, \
                     rows, cols, lost)
  if (side == 128 && tm * tn > kCus) UMEM_SLOPE(128, 1, kPlain);
  else if (side == 128) UMEM_SLOPE(128, 2, kPlain);
  else if (PR == 3 && tm * tn > kCus) UMEM_SLOPE(64, 1, kParts);
  else if (PR == 3) UMEM_SLOPE(64, 2, kParts);
  else if (tm * tn > 2 * kCus) UMEM_SLOPE(64, 1, kPlain);
  else UMEM_SLOPE(64, 2, kPlain);
#undef UMEM_SLOPE
}

}  // namespace

size_t head_loss_workspace_bytes(const umem_head_desc& hd, int T) { return T == 0 ? 0 : ForwardLayout(hd, T).total; }

hipError_t launch_head_loss(const umem_head_desc& hd, int T, const void* x, const uint16_t* w, const int32_t* targets,
                            float* loss, float* lse, void* ws, hipStream_t s) {
  clear_stale_error();
  const ForwardLayout L(hd, T);
  char* base = static_cast<char*>(ws);
  uint16_t* parts = reinterpret_cast<uint16_t*>(base + L.parts);
  float2* stats = reinterpret_cast<float2*>(base + L.stats);
  float* goal = reinterpret_cast<float*>(base + L.goal);
  for (int t0 = 0; t0 < T; t0 += kBandTokens) {
    const int t = std::min(kBandTokens, T - t0);
    const char* xb = static_cast<const char*>(x) + static_cast<size_t>(t0) * hd.d * (hd.xtype == UMEM_F32 ? 4 : 2);
    if (hd.xtype == UMEM_F32) split_x(hd, t, xb, parts, nullptr, nullptr, s);
    const TilePairs p = logit_pairs(hd, t, xb, parts, w, hd.vocab);
    const int side = tile_plan(hd.vocab, t, slice_count(p.k, p.n), 1, true).side;
    const int tiles = (hd.vocab + side - 1) / side, tn = (t + side - 1) / side;
    const double scale = std::fabs(hd.scale / spread_of(hd.scale));
#define UMEM_STATS(BM, WC, GROUPS, PARTS)                                                                        \
  hipLaunchKernelGGL((head_stats_kernel<BM, BM, 2, WC, GROUPS, PARTS>), dim3(tile_grid(tiles * tn)),             \
                     dim3(128 * WC * GROUPS), 0, s, p, tiles, tn, hd.scale, targets + t0, stats, goal)
    if (side == 256) UMEM_STATS(256, 4, 1, kPlain);
    else if (side == 128 && tiles * tn > kCus) UMEM_STATS(128, 2, 1, kPlain);
    else if (side == 128) UMEM_STATS(128, 2, 2, kPlain);
    else if (p.n == 3 && tiles * tn > kCus) UMEM_STATS(64, 2, 1, kThree);
    else if (p.n == 3) UMEM_STATS(64, 2, 2, kThree);
    else if (tiles * tn > 2 * kCus) UMEM_STATS(64, 2, 1, kPlain);
    else UMEM_STATS(64, 2, 2, kPlain);
#undef UMEM_STATS
    if (t <= kFewTokens)
      hipLaunchKernelGGL(head_join_few_kernel, dim3(t), dim3(kThreads), 0, s, stats, goal, targets + t0, t, hd.vocab, tiles,
                         scale, loss + t0, lse + t0);
    else
      hipLaunchKernelGGL(head_join_kernel, dim3((t + 15) / 16), dim3(kThreads), 0, s, stats, goal, targets + t0, t,
                         hd.vocab, tiles, scale, loss + t0, lse + t0);
  }
  return hipGetLastError();
}

size_t head_backward_workspace_bytes(const umem_head_desc& hd, int T) { return T == 0 ? 0 : BackwardLayout(hd, T).total; }

hipError_t launch_head_backward(const umem_head_desc& hd, int T, const void* x, const uint16_t* w, const int32_t* targets,
                                const float* lse, const float* dloss, void* dx, void* dw, bool accumulate, void* ws,
                                hipStream_t s) {
  clear_stale_error();
  const BackwardLayout L(hd, T);
  char* base = static_cast<char*>(ws);
  const auto at = [&](size_t o) { return reinterpret_cast<uint16_t*>(base + o); };
  uint16_t *parts = at(L.parts), *xt = at(L.xt), *wt = at(L.wt), *rows = at(L.rows), *cols = at(L.cols);
  float* sum = reinterpret_cast<float*>(base + L.sum);
  const int d = hd.d, V = hd.vocab, t_pad = static_cast<int>(up(T, 64)), t_ld = static_cast<int>(token_row(T)), piece = piece_rows(hd, T);
  const int pr = row_parts(hd), pc = col_parts(hd), px = x_col_parts(hd);
  const bool wide = hd.xtype == UMEM_F32;
  float* most = dloss ? reinterpret_cast<float*>(base + L.most) : nullptr;
  float* x_most = reinterpret_cast<float*>(base + L.x_most);
  float* lost = reinterpret_cast<float*>(base + L.lost);
  Token* list = reinterpret_cast<Token*>(base + L.list);
  int* count = reinterpret_cast<int*>(base + L.count);
  // x's channels along rows, the tokens that count along k
  const dim3 x_grid(t_pad / 64, (d + 63) / 64);
  if (wide) {
    const float* xf = static_cast<const float*>(x);
    hipLaunchKernelGGL(head_list_kernel<float>, dim3(kMostBlocks), dim3(1024), 0, s, xf, lse, dloss, targets, T, d, V, list,
                       count, most, x_most, static_cast<float*>(dx));
    split_x(hd, T, x, parts, list, count, s);
    const auto turn = px == 2 ? head_transpose_kernel<float, 2> : head_transpose_kernel<float, 1>;
    hipLaunchKernelGGL(turn, x_grid, dim3(kThreads), 0, s, xf, T, d, xt, static_cast<int64_t>(t_ld), x_most, list, count,
                       nullptr);
  } else {
    hipLaunchKernelGGL(head_list_kernel<__bf16>, dim3(kMostBlocks), dim3(1024), 0, s, static_cast<const __bf16*>(x), lse,
                       dloss, targets, T, d, V, list, count, most, x_most, static_cast<__bf16*>(dx));
    hipLaunchKernelGGL((head_transpose_kernel<uint16_t, 1>), x_grid, dim3(kThreads), 0, s,
                       static_cast<const uint16_t*>(x), T, d, xt, static_cast<int64_t>(t_ld), x_most, list, count, parts);
  }
  ProductArgs gx{}, gw{};
  const TilePlan plan_x = dx_plan(hd, T);
  gx.splits = plan_x.splits;
  gx.sums = sum;
  gx.whole = true;
  gx.sum_size = static_cast<int64_t>(T) * d;
  gx.count = gw.count = count;
  gw.along_k = true;
  gw.first = true;
  gw.sums = reinterpret_cast<float*>(base + L.sum_w);
  gx.ld = gw.ld = d;
  gx.most = gw.most = most;
  gw.x_most = x_most;
  gw.scale = hd.scale;
  for (int v0 = 0; v0 < V; v0 += piece) {
    const int v = std::min(piece, V - v0);
    const bool last = v0 + piece >= V;
    const uint16_t* wp = w + static_cast<int64_t>(v0) * d;
    const TilePairs z = logit_pairs(hd, T, parts, parts, wp, v);     // (bf16: the copy of the tokens that count)
    const auto make = pr == 3 ? (pc == 2 ? slope<3, 2> : slope<3, 1>) : (pc == 2 ? slope<1, 2> : slope<1, 1>);
    make(z, hd.scale, list, count, most, v0, piece, t_ld, rows, cols, lost, s);
    // dx: channels along m, tokens along n, the piece along k
    hipLaunchKernelGGL((head_transpose_kernel<uint16_t, 1>), dim3(piece / 64, (d + 63) / 64), dim3(kThreads), 0, s, wp, v,
                       d, wt, static_cast<int64_t>(piece), nullptr, nullptr, nullptr, nullptr);
    TilePairs p{};
    p.n = pr;
    for (int i = 0; i < pr; ++i) {
      p.a[i] = wt;
      p.b[i] = rows + static_cast<int64_t>(pr - 1 - i) * T * piece;
    }
    p.a_rows = d;
    p.b_rows = T;
    p.k = piece;
    p.a_ld = p.b_ld = piece;
    // (without splits the sum of all pieces but the last is kept in `sum` as it is, and scaled with the last)
    gx.first = v0 == 0;
    gx.before = v0 > 0 ? sum : nullptr;
    gx.out = last ? dx : sum;
    gx.scale = last ? hd.scale : 1.f;
    gx.most = last ? most : nullptr;
    gx.list = last ? list : nullptr;
    gx.lost = last && pr == 1 ? lost : nullptr;
    gx.w = w;
    if (!last || wide) product<false, float>(p, gx, plan_x.side, s);
    else product<false, __bf16>(p, gx, plan_x.side, s);
    // dW: channels along m, the piece's rows along n, tokens along k; of fp32 x and two parts of r the pairs that count
    p = TilePairs{};
    const int64_t x_part = static_cast<int64_t>(d) * t_ld, c_part = static_cast<int64_t>(piece) * t_ld;
    for (int i = 2; i >= 0; --i) {
      const int xi = i == 2 ? 1 : 0, ri = i == 1 ? 1 : 0;   // from the smallest products to the largest
      if (xi >= px || ri >= pc) continue;
      p.a[p.n] = xt + xi * x_part;
      p.b[p.n++] = cols + ri * c_part;
    }
    p.a_rows = d;
    p.b_rows = v;
    p.k = t_pad;
    p.a_ld = p.b_ld = t_ld;
    const TilePlan plan_w = dw_plan(hd, T, v);
    const int64_t w_at = static_cast<int64_t>(v0) * d;
    gw.splits = plan_w.splits;
    gw.sum_size = static_cast<int64_t>(v) * d;
    if (hd.gtype == UMEM_F32) {
      float* g = static_cast<float*>(dw) + w_at;
      gw.out = g;
      gw.before = accumulate ? g : nullptr;
      product<true, float>(p, gw, plan_w.side, s);
      if (gw.splits > 1) sum_splits<float>(gw, v, s);
    } else {
      gw.out = static_cast<__bf16*>(dw) + w_at;
      product<true, __bf16>(p, gw, plan_w.side, s);
      if (gw.splits > 1) sum_splits<__bf16>(gw, v, s);
    }
  }
  if (gx.splits > 1) {
    if (wide) sum_splits<float>(gx, T, s);
    else sum_splits<__bf16>(gx, T, s);
  }
  return hipGetLastError();
}

}  // namespace umem
