// The global gradient norm over many tensors, and clipping to it.
//
//   sumsq = sum_i g_i^2,  norm = sqrt(sumsq);   out = g c,  c = 1 if norm <= max else max / norm
//
// Both passes stream: the norm reads every element once, the clip reads and writes it.  The tensors
// travel in the kernel's arguments, up to 64 a launch, so a step's call copies nothing to the GPU and
// can be captured.  A tensor is cut into pieces of one size, a workgroup each; a piece's sum of squares
// is fp64 (the square of a float is exact there, and the conversion and the addition cost less than the
// load), written to its own place and added up in order by one workgroup.
#include <algorithm>

#include "umem_internal.h"

namespace umem {
namespace {

constexpr int THREADS = 256;
constexpr int kTable = 64;                     // tensors in one launch's arguments: 3.6 of 4 KiB
constexpr int64_t kPiece = 8192;               // elements of the smallest piece
constexpr int64_t kPieces = 8192;              // pieces of a call, about, from which they get larger

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

struct Tensor {
  const void* grad;
  void* out;
  const int32_t* n_rows;
  int64_t rows, row_len;
  int32_t bf16;
  int32_t first;                               // its first piece in the launch
};
struct Table {
  Tensor t[kTable];
};
static_assert(sizeof(Tensor) == 48, "the table has to fit the 4 KiB of a kernel's arguments");

// The tensor of piece `b`: the last one that starts at or before it (tensors without elements have no
// pieces and are left out of the table; unused places start past every piece).
__device__ __forceinline__ int tensor_of(const Table& tab, int b) {
  const int lane = threadIdx.x & (kWave - 1);
  const uint64_t before = __ballot(tab.t[lane].first <= b);
  return __builtin_amdgcn_readfirstlane(__popcll(before) - 1);
}

// A piece is [u0, u1) of its tensor's elements counted from the 16-byte boundary at or before the first
// one; the tensor's own elements are [shift, end).
struct Piece {
  int64_t u0, u1, shift, end;
};
__device__ __forceinline__ Piece piece_of(const Tensor& t, int b, int64_t size, int esize) {
  Piece p;
  p.shift = static_cast<int64_t>((reinterpret_cast<uintptr_t>(t.grad) & 15) / esize);
  int64_t rows = t.rows;
  if (t.n_rows != nullptr) rows = min(rows, static_cast<int64_t>(max(*t.n_rows, 0)));
  p.end = rows * t.row_len + p.shift;
  p.u0 = (b - t.first) * size;
  p.u1 = min(p.u0 + size, p.end);
  return p;
}

__device__ __forceinline__ float bf16_lo(uint32_t x) { return __uint_as_float(x << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t x) { return __uint_as_float(x & 0xFFFF0000u); }

__device__ __forceinline__ double wave_sum_f64(double v) {
#pragma unroll
  for (int off = kWave / 2; off > 0; off >>= 1) v += __shfl_xor(v, off, kWave);
  return v;
}

template <typename T>
__device__ __forceinline__ void add_squares(u32x4 x, double (&acc)[4]) {
  if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const double g = static_cast<double>(__uint_as_float(x[i]));
      acc[i] = fma(g, g, acc[i]);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const double lo = static_cast<double>(bf16_lo(x[i])), hi = static_cast<double>(bf16_hi(x[i]));
      acc[i] = fma(lo, lo, acc[i]);
      acc[i] = fma(hi, hi, acc[i]);
    }
  }
}

template <typename T>
__device__ __forceinline__ double piece_squares(const Tensor& t, const Piece& p) {
  constexpr int kPer = 16 / sizeof(T), kDeep = 8;
  const T* base = static_cast<const T*>(t.grad) - p.shift;
  double acc[4] = {0.0, 0.0, 0.0, 0.0};
  const int64_t step = static_cast<int64_t>(THREADS) * kPer;
  int64_t u = p.u0 + static_cast<int64_t>(threadIdx.x) * kPer;
  // whole 16-byte pieces, kDeep in flight a thread
  const int64_t from = max(p.u0, p.shift);
  while (u + (kDeep - 1) * step + kPer <= p.u1 && u >= from) {
    u32x4 x[kDeep];
#pragma unroll
    for (int i = 0; i < kDeep; ++i) x[i] = *reinterpret_cast<const u32x4*>(base + u + i * step);
#pragma unroll
    for (int i = 0; i < kDeep; ++i) add_squares<T>(x[i], acc);
    u += kDeep * step;
  }
  for (; u < p.u1; u += step) {
    if (u >= from && u + kPer <= p.u1) {
      add_squares<T>(*reinterpret_cast<const u32x4*>(base + u), acc);
    } else {
      for (int64_t e = max(u, from); e < min(u + kPer, p.u1); ++e) {
        const double g = static_cast<double>(static_cast<float>(base[e]));
        acc[0] = fma(g, g, acc[0]);
      }
    }
  }
  return (acc[0] + acc[1]) + (acc[2] + acc[3]);
}

__global__ __launch_bounds__(THREADS) void squares_kernel(Table tab, int64_t size, double* part) {
  __shared__ double lds[THREADS / kWave];
  const Tensor& t = tab.t[tensor_of(tab, blockIdx.x)];
  const Piece p = piece_of(t, blockIdx.x, size, t.bf16 ? 2 : 4);
  double s = t.bf16 ? piece_squares<__bf16>(t, p) : piece_squares<float>(t, p);
  s = wave_sum_f64(s);
  if ((threadIdx.x & (kWave - 1)) == 0) lds[threadIdx.x / kWave] = s;
  __syncthreads();
  if (threadIdx.x == 0) part[blockIdx.x] = (lds[0] + lds[1]) + (lds[2] + lds[3]);
}

constexpr int kSumThreads = 1024;
__global__ __launch_bounds__(kSumThreads) void norm_kernel(const double* part, int n, float* norm, double* sumsq) {
  __shared__ double lds[kSumThreads / kWave];
  double s = 0.0;
  for (int i = threadIdx.x; i < n; i += kSumThreads) s += part[i];
  s = wave_sum_f64(s);
  if ((threadIdx.x & (kWave - 1)) == 0) lds[threadIdx.x / kWave] = s;
  __syncthreads();
  if (threadIdx.x != 0) return;
  s = 0.0;
  for (int w = 0; w < kSumThreads / kWave; ++w) s += lds[w];
  *norm = static_cast<float>(sqrt(s));
  if (sumsq != nullptr) *sumsq = s;
}

template <typename T>
__device__ __forceinline__ u32x4 scaled(u32x4 x, float c) {
  u32x4 r;
  if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int i = 0; i < 4; ++i) r[i] = __float_as_uint(__uint_as_float(x[i]) * c);
  } else {
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
#pragma unroll
    for (int i = 0; i < 4; ++i)
      r[i] = __builtin_bit_cast(uint32_t, bf16x2{static_cast<__bf16>(bf16_lo(x[i]) * c),
                                                 static_cast<__bf16>(bf16_hi(x[i]) * c)});
  }
  return r;
}

template <typename T>
__device__ __forceinline__ void piece_scale(const Tensor& t, const Piece& p, float c) {
  constexpr int kPer = 16 / sizeof(T), kDeep = 8;
  const T* in = static_cast<const T*>(t.grad) - p.shift;
  T* out = static_cast<T*>(t.out) - p.shift;
  const int64_t from = max(p.u0, p.shift);
  if (((reinterpret_cast<uintptr_t>(t.grad) ^ reinterpret_cast<uintptr_t>(t.out)) & 15) != 0) {
    // the two lie differently to the 16-byte boundaries: element by element
    for (int64_t e = from + threadIdx.x; e < p.u1; e += THREADS)
      out[e] = static_cast<T>(static_cast<float>(in[e]) * c);
    return;
  }
  const int64_t step = static_cast<int64_t>(THREADS) * kPer;
  int64_t u = p.u0 + static_cast<int64_t>(threadIdx.x) * kPer;
  while (u + (kDeep - 1) * step + kPer <= p.u1 && u >= from) {
    u32x4 x[kDeep];
#pragma unroll
    for (int i = 0; i < kDeep; ++i) x[i] = *reinterpret_cast<const u32x4*>(in + u + i * step);
#pragma unroll
    for (int i = 0; i < kDeep; ++i) *reinterpret_cast<u32x4*>(out + u + i * step) = scaled<T>(x[i], c);
    u += kDeep * step;
  }
  for (; u < p.u1; u += step) {
    if (u >= from && u + kPer <= p.u1) {
      *reinterpret_cast<u32x4*>(out + u) = scaled<T>(*reinterpret_cast<const u32x4*>(in + u), c);
    } else {
      for (int64_t e = max(u, from); e < min(u + kPer, p.u1); ++e)
        out[e] = static_cast<T>(static_cast<float>(in[e]) * c);
    }
  }
}

__global__ __launch_bounds__(THREADS) void clip_kernel(Table tab, int64_t size, float max_norm, const float* norm) {
  const float v = *norm;
  const float c = v <= max_norm ? 1.0f : max_norm / v;
  const Tensor& t = tab.t[tensor_of(tab, blockIdx.x)];
  if (c == 1.0f && t.out == t.grad) return;      // times one in place
  const Piece p = piece_of(t, blockIdx.x, size, t.bf16 ? 2 : 4);
  if (t.bf16) piece_scale<__bf16>(t, p, c);
  else piece_scale<float>(t, p, c);
}

int64_t piece_size(int n, const umem_grad* grads) {
  int64_t total = 0;
  for (int i = 0; i < n; ++i) total += grads[i].rows * grads[i].row_len;
  return std::max<int64_t>(1, (total / kPieces + kPiece - 1) / kPiece) * kPiece;
}

int64_t pieces_of(const umem_grad& g, int64_t size) {
  const int64_t count = g.rows * g.row_len;
  if (count == 0) return 0;
  const int64_t esize = g.dtype == UMEM_BF16 ? 2 : 4;
  const int64_t shift = static_cast<int64_t>((reinterpret_cast<uintptr_t>(g.grad) & 15) / esize);
  return (count + shift + size - 1) / size;
}

// The launches of a call: up to kTable tensors each; go(table, pieces, pieces before them).
template <typename Go>
hipError_t each_table(int n, const umem_grad* grads, int64_t size, Go go) {
  hipError_t e = hipSuccess;
  int64_t before = 0;
  for (int i = 0; i < n && e == hipSuccess;) {
    Table tab;
    int used = 0;
    int64_t pieces = 0;
    for (; i < n && used < kTable; ++i) {
      const int64_t mine = pieces_of(grads[i], size);
      if (mine == 0) continue;
      tab.t[used++] = {grads[i].grad, grads[i].out, grads[i].n_rows, grads[i].rows, grads[i].row_len,
                       grads[i].dtype == UMEM_BF16, static_cast<int32_t>(pieces)};
      pieces += mine;
    }
    if (used == 0) break;
    for (int j = used; j < kTable; ++j) tab.t[j] = {nullptr, nullptr, nullptr, 0, 0, 0, INT32_MAX};
    e = go(tab, static_cast<int>(pieces), before);
    before += pieces;
  }
  return e;
}

}  // namespace

size_t grad_workspace_bytes(int n, const umem_grad* grads) {
  const int64_t size = piece_size(n, grads);
  int64_t pieces = 0;
  for (int i = 0; i < n; ++i) pieces += pieces_of(grads[i], size);
  return (static_cast<size_t>(pieces) * sizeof(double) + 255) / 256 * 256;
}

hipError_t launch_grad_norm(int n, const umem_grad* grads, float* norm, double* sumsq, void* ws, hipStream_t s) {
  clear_stale_error();
  const int64_t size = piece_size(n, grads);
  double* part = static_cast<double*>(ws);
  int64_t total = 0;
  hipError_t e = each_table(n, grads, size, [&](const Table& tab, int pieces, int64_t before) {
    hipLaunchKernelGGL(squares_kernel, dim3(pieces), dim3(THREADS), 0, s, tab, size, part + before);
    total = before + pieces;
    return hipGetLastError();
  });
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(norm_kernel, dim3(1), dim3(kSumThreads), 0, s, part, static_cast<int>(total), norm, sumsq);
  return hipGetLastError();
}

hipError_t launch_grad_clip(int n, const umem_grad* grads, float max_norm, const float* norm, hipStream_t s) {
  clear_stale_error();
  const int64_t size = piece_size(n, grads);
  return each_table(n, grads, size, [&](const Table& tab, int pieces, int64_t) {
    hipLaunchKernelGGL(clip_kernel, dim3(pieces), dim3(THREADS), 0, s, tab, size, max_norm, norm);
    return hipGetLastError();
  });
}

}  // namespace umem
