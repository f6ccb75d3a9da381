// Products of 16-bit matrices on the matrix cores, as the loop that the kernels of the head (head.hip) and of
// the orthogonalised update (orth.hip) share; each brings its own epilogue.
//
//   D[n][m] = sum over parts s, over k of  A_s[m][k] B_s[n][k]        (fp32 sums)
//
// Both operands have k innermost.  A matrix of more bits than 16 is given as parts that add up to it (bf16: three
// hold an fp32 value; fp16: two hold 22 bits of one), and a product of such matrices as the pairs of parts
// that count: the loop walks the pairs one after another over the same accumulators, best from the smallest
// products to the largest, so that these meet no more roundings than alone.
//
// A workgroup takes a tile of BM x BN, its waves in WR x WC blocks of it, K in slices of 64.  What bounds such a
// tile is the matrix cores as long as LDS feeds them: a slice of 256 x 256 x 64 takes the matrix cores 2,048
// clocks and the LDS 1,536 (eight waves of 128 x 64 read 24 KiB each).  Slices go from memory to LDS directly
// (16 bytes a lane), into one of two buffers while the other is read; a row's eight 16-byte pieces lie permuted by its
// number (piece c at place c ^ (row & 7)), so that the lanes that read one piece of eight rows meet all banks.
// The two buffers are arrays of their own: with one array the compiler cannot tell a read of one half from a
// load into the other and waits for the load before each read.
#pragma once

#include "umem_internal.h"

namespace umem {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

constexpr int kTileXcds = 8;
constexpr int kTileBK = 64;             // K's slice: a row's 128 bytes
constexpr int kMaxPairs = 6;

// The parts' pairs of a product.  Rows of ld elements (a multiple of 8), the first k of which count (a multiple of 8);
// every row is 16-byte aligned.  a_rows, b_rows: the rows there are (reads stay below them).
struct TilePairs {
  const uint16_t* a[kMaxPairs];
  const uint16_t* b[kMaxPairs];
  int n;
  int a_rows, b_rows, k;
  int64_t a_ld, b_ld;
};

// What a lane loads in the place of a piece past k.
static __device__ __align__(16) const uint32_t tile_zeros[4] = {0u, 0u, 0u, 0u};

template <bool F16>
__device__ __forceinline__ f32x4 tile_mfma(u32x4 a, u32x4 b, f32x4 c) {
  if constexpr (F16)
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

typedef __attribute__((address_space(3))) uint32_t lds_u32;
typedef const __attribute__((address_space(1))) uint32_t global_u32;

// BM x BN tile of WR x WC waves; acc[a][b]: the 16 x 16 block at m = wave's row + 16 a, n = wave's column + 16 b,
// of which lane l holds m = 4 (l / 16) + 0 .. 3, n = l % 16.
template <bool F16, int BM, int BN, int WR, int WC>
struct Tile {
  static constexpr int kThreads = 64 * WR * WC;
  static constexpr int MT = BM / WR / 16, NT = BN / WC / 16;
  static constexpr int kA = BM * 8 / kThreads, kB = BN * 8 / kThreads;       // 16-byte pieces a thread loads
  static constexpr int kElems = (BM + BN) * kTileBK;                         // one buffer
  static_assert(BM * 8 % kThreads == 0 && BN * 8 % kThreads == 0, "whole pieces");

  uint32_t a_off[kA], b_off[kB];          // a lane's pieces, in bytes from the slice's first
  int col_k;                              // first k of the lane's pieces in a slice, the same for all of them
  int m0, n0;

  // The lane's offsets for the tile at (m0, n0).  A row's number mod 8 is the same for all pieces of a lane
  // (the pieces lie kThreads / 8 rows apart), so their column is too.
  __device__ __forceinline__ void init(const TilePairs& p, int m0_, int n0_) {
    m0 = min(m0_, p.a_rows - 1);            // (a tile past the rows that there are reads the last one)
    n0 = min(n0_, p.b_rows - 1);
    const int tid = threadIdx.x, row = tid >> 3, col = (tid & 7) ^ (row & 7);
    col_k = col * 8;
#pragma unroll
    for (int i = 0; i < kA; ++i) {
      const int r = min(row + i * (kThreads / 8), p.a_rows - 1 - m0);
      a_off[i] = static_cast<uint32_t>(r * static_cast<int>(p.a_ld) + col * 8) * 2u;
    }
#pragma unroll
    for (int i = 0; i < kB; ++i) {
      const int r = min(row + i * (kThreads / 8), p.b_rows - 1 - n0);
      b_off[i] = static_cast<uint32_t>(r * static_cast<int>(p.b_ld) + col * 8) * 2u;
    }
  }

  // A slice into a buffer: the tile's first row of both operands at the slice's first k, k0 of k.
  __device__ __forceinline__ void load(const char* a, const char* b, int k0, int k, uint16_t* lds) const {
    const int wave = threadIdx.x >> 6;
    const bool tail = k0 + kTileBK > k;
    if (!tail) {
#pragma unroll
      for (int i = 0; i < kA; ++i)
        __builtin_amdgcn_global_load_lds((global_u32*)(a + a_off[i]),
                                         (lds_u32*)(lds + (i * kThreads + wave * 64) * 8), 16, 0, 0);
#pragma unroll
      for (int i = 0; i < kB; ++i)
        __builtin_amdgcn_global_load_lds((global_u32*)(b + b_off[i]),
                                         (lds_u32*)(lds + BM * kTileBK + (i * kThreads + wave * 64) * 8), 16, 0, 0);
    } else {
      const bool in = k0 + col_k < k;
      const char* z = reinterpret_cast<const char*>(tile_zeros);
#pragma unroll
      for (int i = 0; i < kA; ++i)
        __builtin_amdgcn_global_load_lds((global_u32*)(in ? a + a_off[i] : z),
                                         (lds_u32*)(lds + (i * kThreads + wave * 64) * 8), 16, 0, 0);
#pragma unroll
      for (int i = 0; i < kB; ++i)
        __builtin_amdgcn_global_load_lds((global_u32*)(in ? b + b_off[i] : z),
                                         (lds_u32*)(lds + BM * kTileBK + (i * kThreads + wave * 64) * 8), 16, 0, 0);
    }
  }

  __device__ __forceinline__ static void compute(const uint16_t* lds, f32x4 (&acc)[MT][NT]) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int wr = wave / WC, wc = wave % WC;
    const int r = lane & 15, q = lane >> 4;
    const uint16_t* a = lds + (wr * MT * 16 + r) * kTileBK;
    const uint16_t* b = lds + BM * kTileBK + (wc * NT * 16 + r) * kTileBK;
#pragma unroll
    for (int kk = 0; kk < 2; ++kk) {
      const int at = ((kk * 4 + q) ^ (r & 7)) * 8;
      u32x4 af[MT], bf[NT];
#pragma unroll
      for (int i = 0; i < NT; ++i) bf[i] = *reinterpret_cast<const u32x4*>(b + i * 16 * kTileBK + at);
#pragma unroll
      for (int i = 0; i < MT; ++i) af[i] = *reinterpret_cast<const u32x4*>(a + i * 16 * kTileBK + at);
#pragma unroll
      for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j) acc[i][j] = tile_mfma<F16>(af[i], bf[j], acc[i][j]);
    }
  }

  // Waits until the loads into LDS of all waves have landed and all have read the other buffer.
  __device__ __forceinline__ static void landed() {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
  }

  // The product over the slices [from, to) of the pairs' slices laid one after another (ceil(k / 64) each).
  __device__ __forceinline__ void run(const TilePairs& p, int from, int to, uint16_t* buf0, uint16_t* buf1,
                                      f32x4 (&acc)[MT][NT]) const {
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
      for (int j = 0; j < NT; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    const int per = (p.k + kTileBK - 1) / kTileBK;
    const int k = p.k;
    int s = from / per, k0 = (from - s * per) * kTileBK;
    const char *a = nullptr, *b = nullptr;
    const auto point = [&] {
      a = reinterpret_cast<const char*>(p.a[s] + m0 * p.a_ld + k0);
      b = reinterpret_cast<const char*>(p.b[s] + n0 * p.b_ld + k0);
    };
    const auto next = [&] {
      k0 += kTileBK;
      a += kTileBK * 2;
      b += kTileBK * 2;
      if (k0 >= k) {
        k0 = 0;
        if (++s < p.n) point();
      }
    };
    point();
    load(a, b, k0, k, buf0);
    int left = to - from;
    while (true) {
      landed();
      next();
      if (left > 1) load(a, b, k0, k, buf1);
      compute(buf0, acc);
      if (--left == 0) break;
      landed();
      next();
      if (left > 1) load(a, b, k0, k, buf0);
      compute(buf1, acc);
      if (--left == 0) break;
    }
  }
};

// The tile that a workgroup takes: the items of one XCD (workgroups go to the XCDs in turn) are consecutive, and run down
// bands of kBand tiles along m, so that the tiles that an XCD works on at once share their operands in its L2.
struct TilePlace {
  int m, n;
};
__device__ __forceinline__ TilePlace tile_place(int item, int tiles_m, int tiles_n) {
  constexpr int kBand = 4;
  const int band = item / (kBand * tiles_n), first = band * kBand;
  const int high = min(kBand, tiles_m - first);
  const int in = item - first * tiles_n;
  return {first + in % high, in / high};
}
__device__ __forceinline__ int tile_item(int items) {
  const int per = (items + kTileXcds - 1) / kTileXcds;
  return (blockIdx.x % kTileXcds) * per + blockIdx.x / kTileXcds;
}
inline int tile_grid(int items) { return (items + kTileXcds - 1) / kTileXcds * kTileXcds; }

}  // namespace umem
