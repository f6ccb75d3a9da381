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
// fp16 matrices of two parts are laid out with both in a row, 32 values' first parts, then their second ones
// (part_at): a slice then holds both parts of 32 values, and a wave takes the three products of them that count from one
// reading of LDS, the two small ones into accumulators of their own (kBoth).
//
// A workgroup takes a tile of BM x BN, its waves in WR x WC blocks of it, K in slices of 64.  What bounds such a
// tile is the matrix cores as long as LDS feeds them: a slice of 256 x 256 x 64 takes the matrix cores 2,048
// clocks and the LDS 1,536 (eight waves of 128 x 64 read 24 KiB each).  Slices go from memory to LDS directly
// (16 bytes a lane), into the buffers after the one that is read, two to four of them; a row's eight 16-byte pieces lie
// permuted by its number (piece c at place c ^ (row & 7)), so that the lanes that read one piece of eight rows meet all
// banks.  The buffers are arrays of their own: within one array the compiler cannot tell a read of one buffer from a
// load into another and waits for the load before each read.
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
constexpr int kMaxPairs = 3;            // three parts of an fp32 value, or three of the four of two values in two parts

// The parts' pairs of a product.  Rows of ld elements (a multiple of 8), the first k of which count (a multiple of 8);
// every row is 16-byte aligned.  a_rows, b_rows: the rows there are (reads stay below them).
struct TilePairs {
  const uint16_t* a[kMaxPairs];
  const uint16_t* b[kMaxPairs];
  int n;
  int a_rows, b_rows, k;
  int64_t a_ld, b_ld;
};

// How k lies in a row: 16-bit values one after another, or both parts of values.  kThree: B is three matrices b[0] to b[2]
// whose products with the one A are added (a value's parts, the smallest first), a slice of all of them at a time, so that
// A passes once: 1,845 x 1,032 tokens over 1,032 34 us a pair after another, so 26.
enum TileParts { kPlain, kBoth, kThree };
// Where a row's value k has its first part (the second is 32 elements on), and the row's elements for k values.
__host__ __device__ __forceinline__ constexpr int64_t part_at(int64_t k) { return (k >> 5) * 64 + (k & 31); }
constexpr int kPartStep = 32;

template <bool F16>
__device__ __forceinline__ f32x4 tile_mfma(u32x4 a, u32x4 b, f32x4 c) {
  if constexpr (F16)
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

typedef __attribute__((address_space(3))) uint32_t lds_u32;

// BM x BN tile of WR x WC waves; acc[a][b]: the 16 x 16 block at m = wave's row + 16 a, n = wave's column + 16 b,
// of which lane l holds m = 4 (l / 16) + 0 .. 3, n = l % 16.
// GROUPS > 1: as many sets of waves, each with buffers of its own, take a share of the slices; the caller adds their
// accumulators.
template <bool F16, int BM, int BN, int WR, int WC, int BUFS, TileParts PARTS = kPlain, int GROUPS = 1>
struct Tile {
  static constexpr int kThreads = 64 * WR * WC;                              // of a group
  static constexpr int MT = BM / WR / 16, NT = BN / WC / 16;
  static constexpr int kA = BM * 8 / kThreads, kB = BN * 8 / kThreads;       // 16-byte pieces a thread loads
  static constexpr int kBs = PARTS == kThree ? 3 : 1, kLoadsOf = kA + kBs * kB;
  static constexpr int kElems = (BM + kBs * BN) * kTileBK;                   // one buffer
  static constexpr int kStep = kTileBK;                                      // a slice's elements of a row
  static constexpr int kAccs = PARTS == kBoth ? 2 : 1;                       // sets of accumulators
  static_assert(BM * 8 % kThreads == 0 && BN * 8 % kThreads == 0, "whole pieces");

  uint32_t a_off[kA], b_off[kB];          // a lane's pieces, in bytes from the tile's first row
  int col_k;                              // first k of the lane's pieces in a slice, the same for all of them
  int m0, n0;

  // The thread within its group, and the group.
  __device__ __forceinline__ static int thread() { return GROUPS == 1 ? threadIdx.x : threadIdx.x % kThreads; }
  __device__ __forceinline__ static int group() {
    return GROUPS == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x / kThreads);
  }

  // The lane's offsets for the tile at (m0, n0).  A row's number mod 8 is the same for all pieces of a lane
  // (the pieces lie kThreads / 8 rows apart), so their column is too.  The tile's row i of A is a_row(i) of the matrix's
  // from m0 on, and so B's: an order of the rows that suits how the caller writes the accumulators.
  struct InOrder {
    __device__ __forceinline__ int operator()(int row) const { return row; }
  };
  template <typename RowA = InOrder, typename RowB = InOrder>
  __device__ __forceinline__ void init(const TilePairs& p, int m0_, int n0_, RowA a_row = {}, RowB b_row = {}) {
    m0 = min(m0_, p.a_rows - 1);            // (a tile past the rows that there are reads the last one)
    n0 = min(n0_, p.b_rows - 1);
    const int tid = thread(), row = tid >> 3, col = (tid & 7) ^ (row & 7);
    col_k = col * 8;
#pragma unroll
    for (int i = 0; i < kA; ++i) {
      const int r = min(a_row(row + i * (kThreads / 8)), p.a_rows - 1 - m0);
      a_off[i] = static_cast<uint32_t>(r * static_cast<int>(p.a_ld) + col_k) * 2u;
    }
#pragma unroll
    for (int i = 0; i < kB; ++i) {
      const int r = min(b_row(row + i * (kThreads / 8)), p.b_rows - 1 - n0);
      b_off[i] = static_cast<uint32_t>(r * static_cast<int>(p.b_ld) + col_k) * 2u;
    }
  }

  // The rows from `row` on, as a buffer.
  __device__ __forceinline__ static __amdgpu_buffer_rsrc_t rows_from(const uint16_t* p, int row, int64_t ld, int rows) {
    const int64_t bytes = (rows - row) * ld * 2;
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<uint16_t*>(p + row * ld), static_cast<short>(0),
                                             static_cast<int>(bytes < 0xffffffffll ? bytes : 0xffffffffll), 0x00020000);
  }

  // The slice from k0 on into a buffer; a piece past k is another one here (past_k).
  __device__ __forceinline__ void load(__amdgpu_buffer_rsrc_t a, const __amdgpu_buffer_rsrc_t (&b)[kBs], int k0, int k,
                                       uint16_t* lds) const {
    const int wave = __builtin_amdgcn_readfirstlane(thread() >> 6);
    const auto get = [&](uint32_t back) {
#pragma unroll
      for (int i = 0; i < kA; ++i)
        __builtin_amdgcn_raw_ptr_buffer_load_lds(a, (lds_u32*)(lds + (i * kThreads + wave * 64) * 8), 16,
                                                 a_off[i] - back, k0 * 2, 0, 0);
#pragma unroll
      for (int s = 0; s < kBs; ++s)
#pragma unroll
        for (int i = 0; i < kB; ++i)
          __builtin_amdgcn_raw_ptr_buffer_load_lds(
              b[s], (lds_u32*)(lds + (BM + s * BN) * kTileBK + (i * kThreads + wave * 64) * 8), 16, b_off[i] - back,
              k0 * 2, 0, 0);
    };
    if (PARTS != kBoth && k0 + kTileBK > k) get(k0 + col_k >= k ? static_cast<uint32_t>(col_k) * 2u : 0u);
    else get(0u);
  }

  // The lane's pieces past k, once they have landed, to zeros.  (Rows of parts are whole slices.)
  __device__ __forceinline__ void past_k(int k0, int k, uint16_t* lds) const {
    if (PARTS == kBoth || k0 + kTileBK <= k) return;
    if (k0 + col_k >= k) {
#pragma unroll
      for (int i = 0; i < kLoadsOf; ++i) {
        uint16_t* piece = lds + (i < kA ? 0 : BM * kTileBK) + ((i < kA ? i : i - kA) * kThreads + thread()) * 8;
        *reinterpret_cast<u32x4*>(piece) = u32x4{0u, 0u, 0u, 0u};
      }
    }
    __builtin_amdgcn_s_waitcnt(0xc07f);                     // lgkmcnt alone
  }

  // A wave's fragments of both halves of a slice, and their products: of halves of k the two that match; of both
  // parts the three that count.
  struct Fragments {
    u32x4 a[2][MT], b[2][NT];
  };
  __device__ __forceinline__ static void read(const uint16_t* lds, int half, Fragments& f) {
    read_b(lds, half, 0, f);
    read_a(lds, half, f);
  }
  __device__ __forceinline__ static void read_a(const uint16_t* lds, int half, Fragments& f) {
    const int lane = threadIdx.x & 63, wave = thread() >> 6;
    const int r = lane & 15, q = lane >> 4, at = ((half * 4 + q) ^ (r & 7)) * 8;
    const uint16_t* a = lds + (wave / WC * MT * 16 + r) * kTileBK;
#pragma unroll
    for (int i = 0; i < MT; ++i) f.a[half][i] = *reinterpret_cast<const u32x4*>(a + i * 16 * kTileBK + at);
  }
  __device__ __forceinline__ static void read_b(const uint16_t* lds, int half, int which, Fragments& f) {
    const int lane = threadIdx.x & 63, wave = thread() >> 6;
    const int r = lane & 15, q = lane >> 4, at = ((half * 4 + q) ^ (r & 7)) * 8;
    const uint16_t* b = lds + (BM + which * BN + wave % WC * NT * 16 + r) * kTileBK;
#pragma unroll
    for (int i = 0; i < NT; ++i) f.b[half][i] = *reinterpret_cast<const u32x4*>(b + i * 16 * kTileBK + at);
  }
  // (With its priority raised meanwhile, a wave's products are not held up by another's reads: 3 to 5 percent.)
  __device__ __forceinline__ static void multiply(const Fragments& f, int x, int y, f32x4 (&acc)[MT][NT]) {
    __builtin_amdgcn_s_setprio(1);
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
      for (int j = 0; j < NT; ++j) acc[i][j] = tile_mfma<F16>(f.a[x][i], f.b[y][j], acc[i][j]);
    __builtin_amdgcn_s_setprio(0);
  }
  // (Reading a slice's fragments while the slice before is multiplied measured the same.)
  __device__ __forceinline__ static void compute(const uint16_t* lds, f32x4 (&acc)[kAccs][MT][NT]) {
    Fragments f;
    if constexpr (PARTS != kThree) read(lds, 0, f);
    if constexpr (PARTS == kBoth) {
      read(lds, 1, f);
      multiply(f, 0, 0, acc[0]);
      multiply(f, 0, 1, acc[kAccs - 1]);
      multiply(f, 1, 0, acc[kAccs - 1]);
    } else if constexpr (PARTS == kThree) {
      // (a part's fragments are read while the ones before are multiplied)
      read(lds, 0, f);
      read_a(lds, 1, f);
#pragma unroll
      for (int s = 0; s < kBs; ++s) {
        read_b(lds, 1, s, f);
        multiply(f, 0, 0, acc[0]);
        if (s + 1 < kBs) read_b(lds, 0, s + 1, f);
        multiply(f, 1, 1, acc[0]);
      }
    } else {
      multiply(f, 0, 0, acc[0]);
      read(lds, 1, f);
      multiply(f, 1, 1, acc[0]);
    }
  }

  // Waits until a wave's loads but for those of the last LATER slices have landed, and until all waves have come here:
  // the slice, at k0 of k in `lds`, is whole, and the buffer before it has been read by everyone.  (A fence would wait
  // for all loads.)
  template <int LATER>
  __device__ __forceinline__ void landed(int k0, int k, uint16_t* lds) const {
    constexpr int kLoads = LATER * kLoadsOf;
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt((kLoads & 15) | (kLoads >> 4) << 14 | 0x0f70);          // vmcnt alone
    past_k(k0, k, lds);
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
  }

  // The slices of p's pairs laid one after another.
  __device__ __forceinline__ static int slices(const TilePairs& p) { return (PARTS == kThree ? 1 : p.n) * ((p.k + kStep - 1) / kStep); }

  // The product over the slices [from, to) of them, to > from (of a group: its share), through BUFS buffers.  Past the last slice that one is
  // loaded again, and the loop has one end: with loads that may or may not be there, and with an exit in its midst, the
  // compiler waits for all loads before a read.  All loads have landed when this returns; all waves have read the last
  // slice only after a barrier.
  __device__ __forceinline__ void run(const TilePairs& p, int from, int to, uint16_t* buf0, uint16_t* buf1,
                                      uint16_t* buf2, uint16_t* buf3, f32x4 (&out)[MT][NT]) const {
    uint16_t* const bufs[4] = {buf0, buf1, buf2, buf3};
    static_assert(BUFS >= 2 && BUFS <= 4 && (BUFS - 2) * kLoadsOf < 64, "what vmcnt counts");
    f32x4 acc[kAccs][MT][NT];
#pragma unroll
    for (int s = 0; s < kAccs; ++s)
#pragma unroll
      for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j) acc[s][i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    // Groups meet at the same barriers: each walks as many slices as the largest share has, and leaves out what is not its own.
    const int share = (to - from + GROUPS - 1) / GROUPS, first = from + group() * share;
    int mine = GROUPS == 1 ? share : min(share, to - first);
    const int k = p.k, per = (k + kStep - 1) / kStep, start = GROUPS == 1 ? first : min(first, to - 1);
    int s = start / per, k0 = (start - s * per) * kStep;    // the next slice to load
    int at = k0;                                            // where in k the next slice to compute lies
    int left = share, ahead = mine;                         // slices to compute, to load
    const uint16_t *pa = nullptr, *pb = nullptr;
    const auto point = [&] {
      pa = p.a[0];
      pb = p.b[0];
#pragma unroll
      for (int i = 1; i < kMaxPairs; ++i) {
        pa = PARTS != kThree && p.n > 1 && s == i ? p.a[i] : pa;
        pb = PARTS != kThree && p.n > 1 && s == i ? p.b[i] : pb;
      }
    };
    const auto fetch = [&](uint16_t* buf) {
      __amdgpu_buffer_rsrc_t b[kBs];
#pragma unroll
      for (int i = 0; i < kBs; ++i) b[i] = rows_from(PARTS == kThree ? p.b[i] : pb, n0, p.b_ld, p.b_rows);
      load(rows_from(pa, m0, p.a_ld, p.a_rows), b, k0, k, buf);
      if (--ahead <= 0) return;
      k0 += kStep;
      if (k0 >= k) {
        k0 = 0;
        ++s;
        point();
      }
    };
    point();
#pragma unroll
    for (int i = 0; i < BUFS - 1; ++i) fetch(bufs[i]);
    for (; left >= BUFS; left -= BUFS) {
#pragma unroll
      for (int i = 0; i < BUFS; ++i) {
        landed<BUFS - 2>(at, k, bufs[i]);                   // in flight: the BUFS - 2 slices after this one
        at = at + kStep >= k ? 0 : at + kStep;
        fetch(bufs[(i + BUFS - 1) % BUFS]);
        if (GROUPS == 1 || mine-- > 0) compute(bufs[i], acc);
      }
    }
    // the last slices, fewer than the buffers, are all there or on their way
#pragma unroll
    for (int i = 0; i < BUFS - 1; ++i) {
      if (i < left) {
        landed<0>(at, k, bufs[i]);
        at = at + kStep >= k ? 0 : at + kStep;
        if (GROUPS == 1 || mine-- > 0) compute(bufs[i], acc);
      }
    }
    __builtin_amdgcn_s_waitcnt(0x0f70);
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
      for (int j = 0; j < NT; ++j) out[i][j] = kAccs == 2 ? acc[0][i][j] + acc[kAccs - 1][i][j] : acc[0][i][j];
  }

  // What each of two groups keeps of the tile for its end, the sums of both: the half of the columns' blocks with its
  // number, through all of a buffer of GROUPS kElems.  (Of one group: everything.)
  static constexpr int NE = NT / (GROUPS > 1 ? 2 : 1);
  __device__ __forceinline__ static void share(const f32x4 (&acc)[MT][NT], uint16_t* lds, f32x4 (&out)[MT][NE]) {
    if constexpr (GROUPS == 1) {
#pragma unroll
      for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j) out[i][j] = acc[i][j];
    } else {
      static_assert(GROUPS == 2 && NT % 2 == 0 && BM * BN * 4 <= GROUPS * kElems * 2, "halves of a tile fit a buffer");
      const int g = group();
      f32x4* const to = reinterpret_cast<f32x4*>(lds) + g * MT * NE * kThreads + thread();
      const f32x4* const from = reinterpret_cast<const f32x4*>(lds) + (1 - g) * MT * NE * kThreads + thread();
      __syncthreads();
#pragma unroll
      for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NE; ++j) to[(i * NE + j) * kThreads] = g == 0 ? acc[i][j + NE] : acc[i][j];
      __syncthreads();
#pragma unroll
      for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NE; ++j) {
          const f32x4 other = from[(i * NE + j) * kThreads], own = g == 0 ? acc[i][j] : acc[i][j + NE];
          out[i][j] = g == 0 ? own + other : other + own;
        }
    }
  }
};

// The tile that a workgroup takes: the items of one XCD (workgroups go to the XCDs in turn) are consecutive, and run down
// bands of kBand tiles along m, so that the tiles that an XCD works on at once share their operands in its L2.
struct TilePlace {
  int m, n;
};
template <int BAND = 4>
__device__ __forceinline__ TilePlace tile_place(int item, int tiles_m, int tiles_n) {
  constexpr int kBand = BAND;
  const int band = item / (kBand * tiles_n), first = band * kBand;
  const int high = min(kBand, tiles_m - first);
  const int in = item - first * tiles_n;
  return {first + in % high, in / high};
}
// (`items`, and past it, of a workgroup without one: a grid may be of more)
__device__ __forceinline__ int tile_item(int items) {
  const int per = (items + kTileXcds - 1) / kTileXcds, in = blockIdx.x / kTileXcds;
  return in < per ? (blockIdx.x % kTileXcds) * per + in : items;
}
inline int tile_grid(int items) { return (items + kTileXcds - 1) / kTileXcds * kTileXcds; }

}  // namespace umem
