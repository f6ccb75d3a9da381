// The global gradient norm over many tensors, and clipping to it.
//
//   sumsq = sum_i g_i^2,  norm = sqrt(sumsq);   out = g c,  c = 1 if norm <= max else max / norm
//
// Both passes stream: the norm reads every element once, the clip reads and writes it, from the last piece to
// the first, so that it begins with what the norm left in the caches.  The tensors travel in the kernel's
// arguments, up to 112 a launch, so a step's call copies nothing to the GPU and can be captured.  A tensor is
// cut into pieces of one size, a workgroup each; a piece's sum of squares is fp64 (the square of a float is
// exact there, and the conversion and the addition cost less than the load), written to its own place and
// added up in order by one workgroup.
//
// Bound by HBM.  The clip's loads and stores are marked as not to be kept: kept in the 256 MB cache, written
// lines were evicted while later kernels read, and 786 MB of gradients took 432 us in both passes together,
// 386 so (norm 125 and clip 251, 6.3 TB/s each; 82 MB 52 and 45 us, 16 MB 20 either way, also with a reader
// of the results behind).  The norm's loads are kept, for the clip: marked as well they made the norm 111 us
// and the clip 272.
#include <algorithm>

#include "umem_internal.h"

namespace umem {
namespace {

constexpr int THREADS = 256;
constexpr int kTable = 112, kCounted = 8;      // tensors in one launch's arguments; with rows counted on the GPU
constexpr int64_t kPiece = 8192;               // elements of the smallest piece
constexpr int64_t kPieces = 8192;              // pieces of a call, about, from which they get larger

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

struct Tensor {
  const void* grad;
  void* out;
  int64_t count;                               // elements; bit 62: of bf16
  int32_t first;                               // its first piece in the launch
  int32_t counted;                             // its place among the counted ones, or -1
};
struct Counted {
  const int32_t* n_rows;
  int64_t rows, row_len;
};
struct Table {
  Tensor t[kTable];
  Counted c[kCounted];
};
constexpr int64_t kBf16 = INT64_C(1) << 62;
static_assert(sizeof(Table) <= 4096 - 256, "the table has to fit the 4 KiB of a kernel's arguments");

// The tensor of piece `b`: the last one that starts at or before it (tensors without elements have no
// pieces and are left out of the table; unused places start past every piece).
__device__ __forceinline__ int tensor_of(const Table& tab, int b) {
  const int lane = threadIdx.x & (kWave - 1);
  const int hi = kWave + lane;
  int before = __popcll(__ballot(tab.t[lane].first <= b));
  before += __popcll(__ballot(hi < kTable && tab.t[min(hi, kTable - 1)].first <= b));
  return __builtin_amdgcn_readfirstlane(before - 1);
}

// A piece is [u0, u1) of its tensor's elements counted from the 16-byte boundary at or before the first
// one; the tensor's own elements are [shift, end).
struct Piece {
  int64_t u0, u1, shift, end;
};
__device__ __forceinline__ Piece piece_of(const Table& tab, const Tensor& t, int b, int64_t size, int esize) {
  Piece p;
  p.shift = static_cast<int64_t>((reinterpret_cast<uintptr_t>(t.grad) & 15) / esize);
  int64_t count = t.count & ~kBf16;
  if (t.counted >= 0) {
    const Counted& c = tab.c[t.counted];
    // (limited before the product, which may not fit 64 bits for a count past the rows there are)
    count = min(static_cast<int64_t>(max(*c.n_rows, 0)), c.rows) * c.row_len;
  }
  p.end = count + p.shift;
  p.u0 = static_cast<int64_t>(b - t.first) * size;
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
  const bool bf16 = (t.count & kBf16) != 0;
  const Piece p = piece_of(tab, t, blockIdx.x, size, bf16 ? 2 : 4);
  double s = bf16 ? piece_squares<__bf16>(t, p) : piece_squares<float>(t, p);
  s = wave_sum_f64(s);
  if ((threadIdx.x & (kWave - 1)) == 0) lds[threadIdx.x / kWave] = s;
  __syncthreads();
  if (threadIdx.x == 0) part[blockIdx.x] = (lds[0] + lds[1]) + (lds[2] + lds[3]);
}

constexpr int kSumThreads = 1024;
__global__ __launch_bounds__(kSumThreads) void norm_kernel(const double* part, int n, float* norm, double* sumsq) {
  __shared__ double lds[kSumThreads / kWave];
  double s = 0.0;
  for (int i0 = threadIdx.x; i0 < n; i0 += 8 * kSumThreads) {
    double v[8];                               // eight in flight, added in order
#pragma unroll
    for (int u = 0; u < 8; ++u) v[u] = i0 + u * kSumThreads < n ? part[i0 + u * kSumThreads] : 0.0;
#pragma unroll
    for (int u = 0; u < 8; ++u) s += v[u];
  }
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
    const T* __restrict__ from_in = in;        // (they are apart, or they would lie alike)
    T* __restrict__ to = out;
#pragma unroll 8
    for (int64_t e = from + threadIdx.x; e < p.u1; e += THREADS)
      to[e] = static_cast<T>(static_cast<float>(from_in[e]) * c);
    return;
  }
  const int64_t step = static_cast<int64_t>(THREADS) * kPer;
  int64_t u = p.u0 + static_cast<int64_t>(threadIdx.x) * kPer;
  while (u + (kDeep - 1) * step + kPer <= p.u1 && u >= from) {
    u32x4 x[kDeep];
#pragma unroll
    for (int i = 0; i < kDeep; ++i) x[i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(in + u + i * step));
#pragma unroll
    for (int i = 0; i < kDeep; ++i) __builtin_nontemporal_store(scaled<T>(x[i], c), reinterpret_cast<u32x4*>(out + u + i * step));
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
  const int b = gridDim.x - 1 - blockIdx.x;
  const Tensor& t = tab.t[tensor_of(tab, b)];
  if (c == 1.0f && t.out == t.grad) return;      // times one in place
  const bool bf16 = (t.count & kBf16) != 0;
  const Piece p = piece_of(tab, t, b, size, bf16 ? 2 : 4);
  if (bf16) piece_scale<__bf16>(t, p, c);
  else piece_scale<float>(t, p, c);
}

int64_t piece_size(int n, const umem_grad* grads) {
  int64_t total = 0;
  for (int i = 0; i < n; ++i) total += grads[i].rows * grads[i].row_len;
  return std::max<int64_t>(1, (total / kPieces + kPiece - 1) / kPiece) * kPiece;
}

// Pieces of a tensor that starts anywhere between two 16-byte boundaries, so that the workspace a program
// sized once does for its gradients wherever they lie.
int64_t pieces_of(const umem_grad& g, int64_t size) {
  const int64_t count = g.rows * g.row_len, shift = g.dtype == UMEM_BF16 ? 7 : 3;
  return count == 0 ? 0 : (count + shift + size - 1) / size;
}

// One launch's tensors: from grads[*i] on, or back from grads[*i - 1], as many as fit, in the list's order.
// Returns their pieces.
int fill_table(const umem_grad* grads, int n, int64_t size, bool back, int* i, Table* tab) {
  int at[kTable], used = 0, counted = 0;
  while (used < kTable && (back ? *i > 0 : *i < n)) {
    const int k = back ? *i - 1 : *i;
    const bool some = pieces_of(grads[k], size) > 0;
    if (some && grads[k].n_rows != nullptr && counted == kCounted) break;
    *i += back ? -1 : 1;
    if (!some) continue;
    counted += grads[k].n_rows != nullptr ? 1 : 0;
    at[used++] = k;
  }
  if (back) std::reverse(at, at + used);
  int pieces = 0, c = 0;
  for (int j = 0; j < used; ++j) {
    const umem_grad& g = grads[at[j]];
    tab->t[j] = {g.grad, g.out, g.rows * g.row_len | (g.dtype == UMEM_BF16 ? kBf16 : 0), pieces, -1};
    if (g.n_rows != nullptr) {
      tab->t[j].counted = c;
      tab->c[c++] = {g.n_rows, g.rows, g.row_len};
    }
    pieces += static_cast<int>(pieces_of(g, size));
  }
  for (int j = used; j < kTable; ++j) tab->t[j] = {nullptr, nullptr, 0, INT32_MAX, -1};
  for (; c < kCounted; ++c) tab->c[c] = {nullptr, 0, 0};
  return pieces;
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
  for (int i = 0; i < n;) {
    Table tab;
    const int pieces = fill_table(grads, n, size, false, &i, &tab);
    if (pieces == 0) break;
    hipLaunchKernelGGL(squares_kernel, dim3(pieces), dim3(THREADS), 0, s, tab, size, part + total);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    total += pieces;
  }
  hipLaunchKernelGGL(norm_kernel, dim3(1), dim3(kSumThreads), 0, s, part, static_cast<int>(total), norm, sumsq);
  return hipGetLastError();
}

hipError_t launch_grad_clip(int n, const umem_grad* grads, float max_norm, const float* norm, hipStream_t s) {
  clear_stale_error();
  const int64_t size = piece_size(n, grads);
  for (int i = n; i > 0;) {
    Table tab;
    const int pieces = fill_table(grads, n, size, true, &i, &tab);
    if (pieces == 0) break;
    hipLaunchKernelGGL(clip_kernel, dim3(pieces), dim3(THREADS), 0, s, tab, size, max_norm, norm);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace umem
