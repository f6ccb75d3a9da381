// Low-rank adapters of many requests beside a shared projection:
//   out[t] = base[t] + scale[i] B_i (A_i x[t]),  i = ids[t];  out[t] = base[t] where i is no adapter
//
// * token_kernel, few tokens (which then mostly have an adapter of their own): a workgroup takes a token
//   and a range of its outputs, both products in one launch.  Bound by the latency of a chain of loads (id,
//   A's rows, B's rows); the ranges recompute A x, whose rows come from L2 after the first, so that few
//   tokens still use many CUs.
// * low_kernel and out_kernel, many tokens: A x on the matrix cores by tiles of 64 tokens and a run of pieces of
//   d_in each, its sums over the runs through the workspace, then B times those by tiles and a range of
//   outputs.  Bound by HBM (x, base and out once, and 8 bytes for each token, rank and run); the adapters come
//   from L2, once for the 16 tokens of a product that share one.  A launch for both, with all of d_in and A for
//   16 tokens in one workgroup, waited for twice as many bytes from L2 in every CU (16 runs, rank 32, 2,048 by
//   896: 1,024 tokens 20.8 us, now 13.7; 4,096 tokens 22, now 20).
//
// Nothing is rounded on the way: an fp32 value is the sum of three bf16 parts of 8 bits each, whose
// products with bf16 weights are exact in the matrix cores' fp32 accumulators.
#include <algorithm>
#include <cmath>

#include "umem_internal.h"

namespace umem {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));

struct AdapterArgs {
  const void* x;
  const int32_t* ids;
  const uint16_t *a, *b;
  const float* scale;
  const void* base;
  void* out;
  int T, n, rank, d_in, d_out;
  int splits;                  // workgroups that share a token's (a tile's) outputs
  float* low;                  // many tokens: [runs of pieces of d_in][T][rank, padded] partial sums of A x
  int runs;                    // runs of pieces of d_in
};

__device__ __forceinline__ float lo_of(uint32_t pair) { return __uint_as_float(pair << 16); }
__device__ __forceinline__ float hi_of(uint32_t pair) { return __uint_as_float(pair & 0xFFFF0000u); }

// Eight consecutive values of x in fp32.
struct Eight {
  float v[8];
};
__device__ __forceinline__ Eight load8(const float* p) {
  const f32x4 a = *reinterpret_cast<const f32x4*>(p), b = *reinterpret_cast<const f32x4*>(p + 4);
  return {{a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w}};
}
__device__ __forceinline__ Eight load8(const __bf16* p) {
  const u32x4 a = *reinterpret_cast<const u32x4*>(p);
  return {{lo_of(a.x), hi_of(a.x), lo_of(a.y), hi_of(a.y), lo_of(a.z), hi_of(a.z), lo_of(a.w), hi_of(a.w)}};
}
__device__ __forceinline__ float dot8(u32x4 w, const Eight& x, float s) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    s = fmaf(lo_of(w[i]), x.v[2 * i], s);
    s = fmaf(hi_of(w[i]), x.v[2 * i + 1], s);
  }
  return s;
}

// ---------------------------------------------------------------- few tokens

// 64 tokens of 64 adapters, rank 16, 1,024 by 2,048: 4.0 us, with 256 or 1,024 threads to a token 4.6.
constexpr int kTokenThreads = 512, kTokenWaves = kTokenThreads / kWave;

// 64 outputs of a token and a wave: L lanes to a row of B, 8 ranks each (lanes past the rank have zeros), so
// that a load is 1,024 consecutive bytes where the rank is 8 L; row u 64 / L + lane / L in load u.  The sums
// over the L lanes leave lane l with output l % L * (64 / L) + l / L.  (A row a lane, with no sums, asks for the same lines L
// times: 256 tokens, rank 64, 2,048 by 2,048: 28.6 us, so 19.)
template <int L, typename OT>
struct Rows64 {
  u32x4 w[L];
  float from;
  static __device__ __forceinline__ int lane() { return threadIdx.x & (kWave - 1); }
  static __device__ __forceinline__ int mine() { return lane() % L * (kWave / L) + lane() / L; }
  // Outputs from o on, those below `last`; b, base: of the token.
  __device__ __forceinline__ void load(const uint16_t* b, const OT* base, int rank, int o, int last) {
    const int q = lane() % L * 8;
#pragma unroll
    for (int u = 0; u < L; ++u) {
      const int row = o + u * (kWave / L) + lane() / L;
      w[u] = u32x4{0, 0, 0, 0};
      if (row < last && q < rank) w[u] = *reinterpret_cast<const u32x4*>(b + static_cast<size_t>(row) * rank + q);
    }
    from = base != nullptr && o + mine() < last ? static_cast<float>(base[o + mine()]) : 0.f;
  }
  __device__ __forceinline__ void store(const Eight& low, OT* out, int o, int last) const {
    float v[L];
#pragma unroll
    for (int u = 0; u < L; ++u) v[u] = dot8(w[u], low, 0.f);
    if constexpr (L >= 16) fold<8, 0x140>(v);          // from the mirrored lane of 16
    if constexpr (L >= 8) fold<4, 0x141>(v);           // of 8
    if constexpr (L >= 4) fold<2, 0x4E>(v);            // from the lane two off
    if constexpr (L >= 2) fold<1, 0xB1>(v);            // one off
    if (o + mine() < last) out[o + mine()] = static_cast<OT>(from + v[0]);
  }
  // Half of the sums go to the partner lane, its half of the others comes back.
  template <int H, int Move>
  static __device__ __forceinline__ void fold(float* v) {
    const bool upper = (lane() & H) != 0;
#pragma unroll
    for (int u = 0; u < H; ++u) {
      const float keep = upper ? v[u + H] : v[u], send = upper ? v[u] : v[u + H];
      v[u] = keep + __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(send), Move, 0xf, 0xf, true));
    }
  }
  // The lane's eight of a token's rank values.
  static __device__ __forceinline__ Eight lows(const float* low, int rank) {
    return lane() % L * 8 < rank ? load8(low + lane() % L * 8) : Eight{};
  }
};

// ROWS: rows of A a wave takes, and the lanes to a row of B: a rank of at most 8 ROWS.
template <typename XT, typename OT, int ROWS>
__global__ __launch_bounds__(kTokenThreads) void token_kernel(AdapterArgs k) {
  __shared__ __align__(16) float low[kMaxAdapterRank];
  const int t = blockIdx.x, part = blockIdx.y;
  const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
  const int id = k.ids[t];
  const bool on = id >= 0 && id < k.n;               // (the same in the whole workgroup)
  // this workgroup's outputs, and this thread's
  const int per = (k.d_out + k.splits - 1) / k.splits, first = part * per, last = min(k.d_out, first + per);
  const OT* base = k.base != nullptr ? static_cast<const OT*>(k.base) + static_cast<size_t>(t) * k.d_out : nullptr;
  OT* out = static_cast<OT*>(k.out) + static_cast<size_t>(t) * k.d_out;
  if (!on) {
    for (int o = first + threadIdx.x; o < last; o += kTokenThreads) out[o] = base != nullptr ? base[o] : OT(0);
    return;
  }
  const uint16_t* b = k.b + static_cast<size_t>(id) * k.d_out * k.rank;
  // kAhead blocks of outputs are loaded together, the first before A x is known
  using Rows = Rows64<ROWS, OT>;
  constexpr int kAhead = ROWS < 8 ? 8 / ROWS : 1;
  Rows even[kAhead], odd[kAhead];
  auto load = [&](Rows* n, int o) {
#pragma unroll
    for (int i = 0; i < kAhead; ++i) n[i].load(b, base, k.rank, o + i * kTokenThreads, last);
  };
  int o = first + wave * kWave;
  load(even, o);
  // A x: a wave's rows side by side, so that its loads of a step are all in flight together
  const XT* x = static_cast<const XT*>(k.x) + static_cast<size_t>(t) * k.d_in;
  const uint16_t* a = k.a + static_cast<size_t>(id) * k.rank * k.d_in;
  float acc[ROWS] = {};
#pragma unroll(ROWS < 8 ? 2 : 1)
  for (int c = lane * 8; c < k.d_in; c += kWave * 8) {
    const Eight xv = load8(x + c);
    u32x4 w[ROWS];
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
      const int row = wave + r * kTokenWaves;
      w[r] = row < k.rank ? *reinterpret_cast<const u32x4*>(a + static_cast<size_t>(row) * k.d_in + c) : u32x4{0, 0, 0, 0};
    }
#pragma unroll
    for (int r = 0; r < ROWS; ++r) acc[r] = dot8(w[r], xv, acc[r]);
  }
  const float scale = k.scale != nullptr ? k.scale[id] : 1.0f;
#pragma unroll
  for (int r = 0; r < ROWS; ++r) {
    const float s = wave_sum(acc[r]);
    if (lane == 0) low[wave + r * kTokenWaves] = s * scale;
  }
  __syncthreads();
  const Eight lows = Rows::lows(low, k.rank);
  auto finish = [&](const Rows* n, int o) {
#pragma unroll
    for (int i = 0; i < kAhead; ++i) n[i].store(lows, out, o + i * kTokenThreads, last);
  };
  constexpr int kStep = kAhead * kTokenThreads;
  for (; o < last; o += 2 * kStep) {
    if (o + kStep < last) load(odd, o + kStep);
    finish(even, o);
    if (o + kStep >= last) break;
    if (o + 2 * kStep < last) load(even, o + 2 * kStep);
    finish(odd, o + kStep);
  }
}

// ---------------------------------------------------------------- many tokens

constexpr int kThreads = 512, kWaves = kThreads / kWave;
constexpr int kTile = 64, kGroup = 16;       // tokens of a workgroup, and of a matrix product

// x = p[0] + p[1] + p[2], each of 8 significant bits (cut off, not rounded, so that the largest values stay
// finite); an infinity is its first part alone.  Four values as three times four bf16.
struct Parts4 {
  u32x2 p[3];
};
__device__ __forceinline__ Parts4 split4(f32x4 x) {
  uint32_t bits[3][4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float rest = x[i];
#pragma unroll
    for (int q = 0; q < 3; ++q) {
      const uint32_t cut = __float_as_uint(rest) & 0xFFFF0000u;
      bits[q][i] = cut;
      rest -= __uint_as_float(cut);
      if (q == 0) rest = fabsf(x[i]) == INFINITY ? 0.f : rest;
    }
  }
  Parts4 r;
#pragma unroll
  for (int q = 0; q < 3; ++q) r.p[q] = u32x2{(bits[q][0] >> 16) | bits[q][1], (bits[q][2] >> 16) | bits[q][3]};
  return r;
}

// An infinite weight meets the zeros among the parts of an ordinary value: a sum that comes out NaN is taken again
// from the values themselves, so that it is what the formula gives, however many tokens there are.  (Until all four
// sums of a lane are NaN, so a NaN among the values ends it.)
__device__ __forceinline__ bool any_nan(f32x4 x) {
  return x.x != x.x || x.y != x.y || x.z != x.z || x.w != x.w;
}
__device__ __forceinline__ bool all_nan(f32x4 x) {
  return x.x != x.x && x.y != x.y && x.z != x.z && x.w != x.w;
}

// Buffer resource of a raw byte range: loads past it give zeros, stores past it are dropped, so the edges
// (tokens past T, ranks past the rank, columns past a width) need no branches around loads and stores.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t rsrc(const void* p, size_t bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), static_cast<short>(0), static_cast<int>(bytes), 0x00020000);
}
constexpr uint32_t kOutside = 0x80000000u;   // past any range here (they are below 2^26 bytes)
__device__ __forceinline__ u32x4 fetch16(__amdgpu_buffer_rsrc_t r, uint32_t at) {
  return __builtin_amdgcn_raw_buffer_load_b128(r, at, 0, 0);
}

// The tokens of a tile, one a lane, and the (span, adapter) pairs among them, a span being 16 CG tokens: the
// first token of each adapter in its span stands for the pair.
template <int CG>
struct Tile {
  static constexpr int kSpan = kGroup * CG;
  int id;                    // this lane's token's adapter, or -1
  uint64_t leads;
  // The id is fetched before a kernel's other loads (they come back in order), and looked at after.
  __device__ __forceinline__ void fetch(const int32_t* ids, int t0, int T) {
    const int t = t0 + (threadIdx.x & (kWave - 1));
    id = t < T ? ids[t] : -1;
  }
  __device__ __forceinline__ void find(int n) {
    if (id < 0 || id >= n) id = -1;
    if constexpr (CG == 1) {       // 16 lanes are a row of the data-parallel moves
      bool first = id >= 0;
      earlier<1>(first);
      leads = __ballot(first);
    } else {
      leads = 0;
      const uint64_t on = __ballot(id >= 0);
#pragma unroll
      for (int c = 0; c < kTile / kSpan; ++c) {
        for (uint64_t left = on & (~0ull >> (kTile - kSpan)) << (c * kSpan); left != 0;) {
          const int first = __builtin_ctzll(left);
          leads |= 1ull << first;
          left &= ~__ballot(id == __builtin_amdgcn_readlane(id, first));
        }
      }
    }
  }
  template <int S>
  __device__ __forceinline__ void earlier(bool& first) {
    // the id S lanes back in the row of 16; past its start -1, which is no adapter
    first = first && __builtin_amdgcn_update_dpp(-1, id, 0x110 + S, 0xf, 0xf, false) != id;
    if constexpr (S < 15) earlier<S + 1>(first);
  }
  // The place of pair p's first token.
  __device__ __forceinline__ int place(int p) const {
    const int lane = threadIdx.x & (kWave - 1);
    const bool it = ((leads >> lane) & 1) != 0 && __popcll(leads & lanemask_lt()) == p;
    return __builtin_ctzll(__ballot(it));
  }
  // Whether the token of this lane's column in the 16 from `first` on has adapter `lead`.
  __device__ __forceinline__ bool mine(int first, int lead) const {
    return __shfl(id, first + (threadIdx.x & (kGroup - 1)), kWave) == lead;
  }
};

// A 16 x 16 x 32 product takes its first operand's rows and its second's columns from lanes % 16, eight
// consecutive k from lane / 16; lane % 16 of the result is its column, and the lane holds rows
// 4 (lane / 16) + 0..3 of it.  The weights are the rows (ranks, then outputs), tokens the columns, so that a
// lane ends up with four consecutive values of one token; columns of tokens with another adapter are
// computed along and dropped (a token's values reach no other column).

// low[run][t][:] = A x over the columns of a run of `walk` pieces.  x of the tile and a piece is staged in LDS in bf16
// parts; a wave takes (pair, 16 ranks) items, whose weights go from global memory to its registers, the next item's
// while this one is multiplied.  NB: 16-byte pieces of x that a thread stages.  RT: rank / 16, rounded up.
// CG: products that share loaded weights; 1 up to rank 32, where a tile of one adapter would leave waves
// without an item, 2 beyond (rank 64, 2,048 by 2,048: 13.8 us, not 16.5).
// WALK: more than one piece.  A wave's items are the same in each, so a lane adds to the sums that it wrote itself.
// (The next piece's x fetched before this one is multiplied: 142 to 174 registers for bf16, one workgroup to a CU, and
// slower in fp32 as well, 487 us where 481 are; so four waves a SIMD, and the other workgroup's work in between.)
template <typename XT>
constexpr int piece_width(int nb) {
  return nb * kThreads / kTile * static_cast<int>(16 / sizeof(XT));
}

template <typename XT, int NB, int CG, bool WALK>
__global__ __launch_bounds__(kThreads, WALK ? 4 : 1) void low_kernel(AdapterArgs k, int RT, int walk) {
  constexpr int kParts = sizeof(XT) == 4 ? 3 : 1, kPer = 16 / sizeof(XT), kPiece = piece_width<XT>(NB);
  constexpr int kPitch = kPiece + 8, kPlane = kTile * kPitch, kSteps = kPiece / 32, kPerRow = kPiece / kPer;
  extern __shared__ __align__(16) uint16_t staged[];    // [parts][64][pitch]
  const int t0 = blockIdx.x * kTile;
  int begin = blockIdx.y * (WALK ? walk * kPiece : kPiece), width = min(kPiece, k.d_in - begin);
  const int end = WALK ? min(begin + walk * kPiece, k.d_in) : 0;
  bool more = false;                                    // whether sums of the run's earlier pieces are there
  const int lane = threadIdx.x & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int col = lane & 15, quad = lane >> 4;
  const int tokens = min(kTile, k.T - t0);
  const size_t row = static_cast<size_t>(k.d_in) * sizeof(XT);
  const __amdgpu_buffer_rsrc_t rx = rsrc(static_cast<const XT*>(k.x) + static_cast<size_t>(t0) * k.d_in, tokens * row);
  Tile<CG> tile;
  tile.fetch(k.ids, t0, k.T);
  // an item's weights in one or two halves of 8 steps, or those of two items of two steps: up to 32 registers at
  // a time, so that two workgroups fit a CU
  constexpr int kHalf = kSteps < 8 ? kSteps : 8, kHalves = kSteps / kHalf, kItems = kHalf < 4 ? 2 : 1;
  static_assert(kParts == 1 || kHalves == 1, "a sum that is taken again starts from its own half's");
  int items = 0;
  struct Half {
    int first[kItems], lead[kItems], rt[kItems];
    u32x4 w[kItems][kHalf];
    f32x4 sums[WALK ? kItems : 1][CG];
  } even, odd;
  // this lane's four sums of an item's tokens from `first` on
  auto sums_at = [&](int first, int rt) {
    return reinterpret_cast<f32x4*>(k.low + ((static_cast<size_t>(blockIdx.y) * k.T + t0 + first + col) * RT + rt) * 16 + quad * 4);
  };
  auto item_of = [&](int half, int i) { return wave + (half / kHalves * kItems + i) * kWaves; };
  auto load = [&](Half& n, int half) {                  // (the wave's own count of halves)
    const int from_step = half % kHalves * kHalf;
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
      const int item = item_of(half, i);
      if (item >= items) return;
      const int pair = item / RT;
      const int at = tile.place(pair);
      n.rt[i] = item - pair * RT;
      n.first[i] = at & ~(Tile<CG>::kSpan - 1);
      n.lead[i] = __builtin_amdgcn_readlane(tile.id, at);
      const __amdgpu_buffer_rsrc_t ra = rsrc(k.a + static_cast<size_t>(n.lead[i]) * k.rank * k.d_in,
                                             static_cast<size_t>(k.rank) * k.d_in * 2);
      const int at_k = from_step * 32 + quad * 8;
      const uint32_t from = static_cast<uint32_t>((n.rt[i] * 16 + col) * k.d_in + begin + at_k) * 2u;
#pragma unroll
      for (int s = 0; s < kHalf; ++s)
        n.w[i][s] = fetch16(ra, s * 32 + at_k < width ? from + static_cast<uint32_t>(s) * 64u : kOutside);
      if constexpr (WALK) {
        if (from_step != 0) continue;
#pragma unroll
        for (int c = 0; c < CG; ++c) {
          const int first = n.first[i] + c * kGroup;
          n.sums[i][c] = f32x4{0.f, 0.f, 0.f, 0.f};
          if (more && tile.mine(first, n.lead[i])) n.sums[i][c] = *sums_at(first, n.rt[i]);
        }
      }
    }
  };
  f32x4 acc[CG];
  auto finish = [&](const Half& n, int half) {
    const int from_step = half % kHalves * kHalf;
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
      if (item_of(half, i) >= items) return;
      const uint16_t* xs = staged + (n.first[i] + col) * kPitch + from_step * 32 + quad * 8;
      if (from_step == 0) {
#pragma unroll
        for (int c = 0; c < CG; ++c) acc[c] = WALK ? n.sums[i][c] : f32x4{0.f, 0.f, 0.f, 0.f};
      }
#pragma unroll
      for (int s = 0; s < kHalf; ++s)
#pragma unroll
        for (int q = 0; q < kParts; ++q)
#pragma unroll
          for (int c = 0; c < CG; ++c)
            acc[c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                __builtin_bit_cast(bf16x8, n.w[i][s]),
                *reinterpret_cast<const bf16x8*>(xs + q * kPlane + c * kGroup * kPitch + s * 32), acc[c], 0, 0, 0);
      if (from_step + kHalf != kSteps) return;
#pragma unroll
      for (int c = 0; c < CG; ++c) {
        const int first = n.first[i] + c * kGroup;
        if (!tile.mine(first, n.lead[i])) continue;
        if (kParts > 1 && any_nan(acc[c])) {
          const int r0 = n.rt[i] * 16 + quad * 4;       // (of padded ranks nothing is read)
          f32x4 s = WALK ? n.sums[i][c] : f32x4{0.f, 0.f, 0.f, 0.f};
          if (r0 < k.rank) {
            const XT* x = static_cast<const XT*>(k.x) + static_cast<size_t>(t0 + first + col) * k.d_in + begin;
            const uint16_t* a = k.a + (static_cast<size_t>(n.lead[i]) * k.rank + r0) * k.d_in + begin;
#pragma unroll 1
            for (int j = 0; j < width && !all_nan(s); ++j)
#pragma unroll
              for (int r = 0; r < 4; ++r) s[r] = fmaf(lo_of(a[static_cast<size_t>(r) * k.d_in + j]), static_cast<float>(x[j]), s[r]);
          }
          acc[c] = s;
        }
        *sums_at(first, n.rt[i]) = acc[c];
      }
    }
  };
  for (;;) {
    u32x4 v[NB];
#pragma unroll
    for (int u = 0; u < NB; ++u) {
      const int f = threadIdx.x + u * kThreads, r = f / kPerRow, c = f % kPerRow * kPer;
      v[u] = fetch16(rx, c < width ? static_cast<uint32_t>(r * k.d_in + begin + c) * static_cast<uint32_t>(sizeof(XT)) : kOutside);
    }
    if (!more) {
      tile.find(k.n);
      if (tile.leads == 0) return;                      // (the same in every wave)
      items = __popcll(tile.leads) * RT;
    }
    load(even, 0);
    if (more) __syncthreads();                          // no wave reads the last piece any more
#pragma unroll
    for (int u = 0; u < NB; ++u) {
      const int f = threadIdx.x + u * kThreads, r = f / kPerRow, c = f % kPerRow * kPer;
      if constexpr (kParts == 1) {
        *reinterpret_cast<u32x4*>(staged + r * kPitch + c) = v[u];
      } else {
        const Parts4 s = split4(__builtin_bit_cast(f32x4, v[u]));
#pragma unroll
        for (int q = 0; q < 3; ++q) *reinterpret_cast<u32x2*>(staged + q * kPlane + r * kPitch + c) = s.p[q];
      }
    }
    __syncthreads();
    for (int half = 0; item_of(half, 0) < items; half += 2) {
      load(odd, half + 1);
      finish(even, half);
      load(even, half + 2);
      finish(odd, half + 1);
    }
    if constexpr (!WALK) return;
    begin += kPiece;
    if (begin >= end) return;
    width = min(kPiece, k.d_in - begin);
    more = true;
  }
}

// Four values of base and out.
template <typename OT>
struct Quad4;
template <>
struct Quad4<float> {
  u32x4 raw;
  __device__ __forceinline__ void load(__amdgpu_buffer_rsrc_t r, uint32_t at) { raw = fetch16(r, at); }
  __device__ __forceinline__ void store(__amdgpu_buffer_rsrc_t r, uint32_t at) const {
    __builtin_amdgcn_raw_buffer_store_b128(raw, r, at, 0, 0);
  }
  __device__ __forceinline__ void add_store(__amdgpu_buffer_rsrc_t r, uint32_t at, f32x4 d) const {
    const f32x4 v = __builtin_bit_cast(f32x4, raw) + d;
    __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, v), r, at, 0, 0);
  }
};
template <>
struct Quad4<__bf16> {
  u32x2 raw;
  __device__ __forceinline__ void load(__amdgpu_buffer_rsrc_t r, uint32_t at) {
    raw = __builtin_amdgcn_raw_buffer_load_b64(r, at, 0, 0);
  }
  __device__ __forceinline__ void store(__amdgpu_buffer_rsrc_t r, uint32_t at) const {
    __builtin_amdgcn_raw_buffer_store_b64(raw, r, at, 0, 0);
  }
  __device__ __forceinline__ void add_store(__amdgpu_buffer_rsrc_t r, uint32_t at, f32x4 d) const {
    const f32x4 v = f32x4{lo_of(raw.x), hi_of(raw.x), lo_of(raw.y), hi_of(raw.y)} + d;
    const bf16x4 o = {static_cast<__bf16>(v.x), static_cast<__bf16>(v.y), static_cast<__bf16>(v.z), static_cast<__bf16>(v.w)};
    __builtin_amdgcn_raw_buffer_store_b64(__builtin_bit_cast(u32x2, o), r, at, 0, 0);
  }
};

// out = base + B (scale low), a tile of tokens and a range of outputs a workgroup.  The runs' sums are
// added in order as they are staged.  KT: steps of 32 over the rank.
//
// Where at least two tokens share an adapter on average, a wave takes units of a pair and 16 U outputs on the
// matrix cores, a unit's loads in flight while the one before is multiplied; else (a batch of many adapters in no
// order) the products would compute 16 columns for one or two, and by_token does it.  Rank 32, 2,048 by 896,
// 2,048 tokens: of 8 adapters in random order (28 pairs) 13.6 us, by token 19.6; of 64 (55 pairs) 24, by token
// 21.  Rank 64, 2,048 by 2,048, 512 tokens of 64 in random order: by token 33, an output a lane 47.
constexpr int kManyPairs = kTile / 2;

// The wave's tokens of a tile (every eighth), a token and kBlocks times 64 outputs at a time.  ids: the tile's, a lane each.
template <int L, typename OT>
__device__ __forceinline__ void by_token(const AdapterArgs& k, const float* low, int pitch, int ids, int t0, int tokens,
                                         int wave, int begin, int end) {
  using Rows = Rows64<L, OT>;
  constexpr int kBlocks = L < 4 ? 4 / L : 1, kStep = kBlocks * kWave;
  const int blocks = (end - begin + kStep - 1) / kStep;
  const int units = blocks > 0 ? (tokens - wave + kWaves - 1) / kWaves * blocks : 0;
  struct Unit {
    Rows rows[kBlocks];
    int tok, o;
    bool on;
  } even, odd;
  auto load = [&](Unit& n, int unit) {
    n.on = unit < units;
    if (!n.on) return;
    n.tok = wave + unit / blocks * kWaves;
    n.o = begin + unit % blocks * kStep;
    const int id = __builtin_amdgcn_readlane(ids, n.tok);
    n.on = id >= 0;
    if (!n.on) return;
    const uint16_t* b = k.b + static_cast<size_t>(id) * k.d_out * k.rank;
    const OT* base = k.base != nullptr ? static_cast<const OT*>(k.base) + static_cast<size_t>(t0 + n.tok) * k.d_out : nullptr;
#pragma unroll
    for (int i = 0; i < kBlocks; ++i) n.rows[i].load(b, base, k.rank, n.o + i * kWave, end);
  };
  auto finish = [&](const Unit& n) {
    if (!n.on) return;
    OT* out = static_cast<OT*>(k.out) + static_cast<size_t>(t0 + n.tok) * k.d_out;
    const Eight lows = Rows::lows(low + n.tok * pitch, k.rank);
#pragma unroll
    for (int i = 0; i < kBlocks; ++i) n.rows[i].store(lows, out, n.o + i * kWave, end);
  };
  load(even, 0);
  for (int unit = 0; unit < units; unit += 2) {
    load(odd, unit + 1);
    finish(even);
    load(even, unit + 2);
    finish(odd);
  }
}

template <typename OT, int KT>
__global__ __launch_bounds__(kThreads) void out_kernel(AdapterArgs k, int RT) {
  constexpr int CG = KT == 1 ? 1 : 2, U = KT == 1 ? 4 : KT == 2 ? 2 : 1;
  constexpr int kPitch = KT * 32 + 8, kPlane = kTile * kPitch;
  __shared__ __align__(16) uint16_t staged[3 * kPlane];
  float* plain = reinterpret_cast<float*>(staged);      // with many pairs: [64][32 KT] in fp32
  static_assert(kTile * KT * 8 == KT * kThreads && kTile * KT * 32 * 4 <= 3 * kPlane * 2, "the plain values take the place of the parts");
  const int t0 = blockIdx.x * kTile;
  const int lane = threadIdx.x & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int col = lane & 15, quad = lane >> 4;
  const int tokens = min(kTile, k.T - t0);
  // this workgroup's output tiles of 16
  const int n_out = (k.d_out + 15) / 16, per = (n_out + k.splits - 1) / k.splits;
  const int o_begin = blockIdx.y * per, o_end = min(n_out, o_begin + per);
  Tile<CG> tile;
  tile.fetch(k.ids, t0, k.T);
  // the rank values of a token are pieces of four; ranks past the rank are zeros.  (Tokens without an adapter
  // have none: what the workspace holds there goes nowhere.)
  f32x4 low[KT];
#pragma unroll
  for (int u = 0; u < KT; ++u) {
    const int f = threadIdx.x + u * kThreads, tok = f / (KT * 8), r4 = f % (KT * 8);
    low[u] = f32x4{0.f, 0.f, 0.f, 0.f};
    if (tok < tokens && r4 * 4 < k.rank) {
      const float* p = k.low + (static_cast<size_t>(t0 + tok) * RT * 4 + r4) * 4;
      const size_t stride = static_cast<size_t>(k.T) * RT * 16;
#pragma unroll 8
      for (int i = 0; i < k.runs; ++i) low[u] += *reinterpret_cast<const f32x4*>(p + i * stride);
    }
  }
  tile.find(k.n);
  const int pairs = __popcll(tile.leads);
  const bool many = pairs > kManyPairs;
  const size_t row = static_cast<size_t>(k.d_out) * sizeof(OT);
  const __amdgpu_buffer_rsrc_t rout = rsrc(static_cast<OT*>(k.out) + static_cast<size_t>(t0) * k.d_out, tokens * row);
  // no base: an empty range, which reads as zeros
  const __amdgpu_buffer_rsrc_t rbase =
      k.base != nullptr ? rsrc(static_cast<const OT*>(k.base) + static_cast<size_t>(t0) * k.d_out, tokens * row)
                        : rsrc(k.out, 0);
  // the units, pair by pair, in equal runs for the waves
  const int blocks = (max(0, o_end - o_begin) + U - 1) / U, units = pairs * blocks;
  const int u_begin = units * wave / kWaves, u_end = units * (wave + 1) / kWaves;
  struct Unit {
    u32x4 w[U][KT];
    Quad4<OT> from[U][CG];
    int first, lead, o;
  } even, odd;
  auto offset = [&](const Unit& n, int u, int c) {
    const int at = (n.o + u) * 16 + quad * 4, first = n.first + c * kGroup;
    return tile.mine(first, n.lead) && n.o + u < o_end && at < k.d_out
               ? static_cast<uint32_t>((first + col) * k.d_out + at) * static_cast<uint32_t>(sizeof(OT)) : kOutside;
  };
  auto load = [&](Unit& n, int unit) {
    if (unit >= u_end) return;
    const int pair = unit / blocks, place = tile.place(pair);
    n.lead = __builtin_amdgcn_readlane(tile.id, place);
    n.first = place & ~(Tile<CG>::kSpan - 1);
    n.o = o_begin + (unit - pair * blocks) * U;
    const __amdgpu_buffer_rsrc_t rb = rsrc(k.b + static_cast<size_t>(n.lead) * k.d_out * k.rank,
                                           static_cast<size_t>(k.d_out) * k.rank * 2);
#pragma unroll
    for (int u = 0; u < U; ++u) {
#pragma unroll
      for (int s = 0; s < KT; ++s) {
        const int kk = s * 32 + quad * 8;
        n.w[u][s] = fetch16(rb, kk < k.rank && n.o + u < o_end ? static_cast<uint32_t>(((n.o + u) * 16 + col) * k.rank + kk) * 2u : kOutside);
      }
#pragma unroll
      for (int c = 0; c < CG; ++c) n.from[u][c].load(rbase, offset(n, u, c));
    }
  };
  // the first unit's loads, before the rank values are there
  if (!many) load(even, u_begin);
#pragma unroll
  for (int u = 0; u < KT; ++u) {
    const int f = threadIdx.x + u * kThreads, tok = f / (KT * 8), r4 = f % (KT * 8);
    const int id = __shfl(tile.id, tok, kWave);
    if (k.scale != nullptr && id >= 0) low[u] *= k.scale[id];
    if (many) {
      *reinterpret_cast<f32x4*>(plain + tok * KT * 32 + r4 * 4) = low[u];
    } else {
      const Parts4 s = split4(low[u]);
#pragma unroll
      for (int q = 0; q < 3; ++q) *reinterpret_cast<u32x2*>(staged + q * kPlane + tok * kPitch + r4 * 4) = s.p[q];
    }
  }
  // tokens without an adapter
  const uint64_t none = __ballot(tile.id < 0 && lane < tokens);
  if (none != 0) {
    for (int tok = wave; tok < tokens; tok += kWaves) {
      if (((none >> tok) & 1) == 0) continue;
      for (int o = o_begin * 16 + lane * 4; o < min(o_end * 16, k.d_out); o += kWave * 4) {
        const uint32_t off = static_cast<uint32_t>(tok * k.d_out + o) * static_cast<uint32_t>(sizeof(OT));
        Quad4<OT> from;
        from.load(rbase, off);
        from.store(rout, off);
      }
    }
  }
  __syncthreads();
  if (many) {
    if constexpr (KT == 1) {
      if (k.rank <= 8) by_token<1, OT>(k, plain, KT * 32, tile.id, t0, tokens, wave, o_begin * 16, min(o_end * 16, k.d_out));
      else if (k.rank <= 16) by_token<2, OT>(k, plain, KT * 32, tile.id, t0, tokens, wave, o_begin * 16, min(o_end * 16, k.d_out));
      else by_token<4, OT>(k, plain, KT * 32, tile.id, t0, tokens, wave, o_begin * 16, min(o_end * 16, k.d_out));
    } else {
      by_token<KT * 4, OT>(k, plain, KT * 32, tile.id, t0, tokens, wave, o_begin * 16, min(o_end * 16, k.d_out));
    }
    return;
  }
  auto finish = [&](const Unit& n, int unit) {
    if (unit >= u_end) return;
#pragma unroll
    for (int c = 0; c < CG; ++c) {
      const uint16_t* p = staged + (n.first + c * kGroup + col) * kPitch + quad * 8;
      bf16x8 v[KT][3];
#pragma unroll
      for (int s = 0; s < KT; ++s)
#pragma unroll
        for (int q = 0; q < 3; ++q) v[s][q] = *reinterpret_cast<const bf16x8*>(p + q * kPlane + s * 32);
#pragma unroll
      for (int u = 0; u < U; ++u) {
        f32x4 d = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int s = 0; s < KT; ++s)
#pragma unroll
          for (int q = 2; q >= 0; --q)
            d = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, n.w[u][s]), v[s][q], d, 0, 0, 0);
        const uint32_t at = offset(n, u, c);
        if (at != kOutside && any_nan(d)) {
          const uint16_t* v = staged + (n.first + c * kGroup + col) * kPitch;
          const uint16_t* b = k.b + (static_cast<size_t>(n.lead) * k.d_out + (n.o + u) * 16 + quad * 4) * k.rank;
          d = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll 1
          for (int j = 0; j < k.rank && !all_nan(d); ++j) {
            const float x = lo_of(v[j]) + (lo_of(v[kPlane + j]) + lo_of(v[2 * kPlane + j]));
#pragma unroll
            for (int r = 0; r < 4; ++r) d[r] = fmaf(lo_of(b[r * k.rank + j]), x, d[r]);
          }
        }
        n.from[u][c].add_store(rout, at, d);
      }
    }
  };
  for (int unit = u_begin; unit < u_end; unit += 2) {
    load(odd, unit + 1);
    finish(even, unit);
    load(even, unit + 2);
    finish(odd, unit + 1);
  }
}

// Tiles of 64 from this many ranks of tokens on (2,560 tokens of rank 16, 640 of rank 64).  A workgroup a token
// does its own A x whoever shares the adapter, a tile shares it, but only among tokens that lie together, and
// has few workgroups.  In us, a workgroup a token and tiles, for 8 adapters in runs, 64 in runs, 64 in random
// order (only the device knows it; what n alone says of the sharing is not used): rank 16, 1,024 by 2,048: 2,048
// tokens 20, 21, 25 and 16, 16, 30; 4,096 36, 36, 44 and 20, 21, 48.  Rank 32, 2,048 by 896: 1,024 tokens
// 16, 20, 24 and 14, 15, 40; 2,048 28, 27, 43 and 15, 17, 53.  Rank 64, 2,048 by 2,048: 512 tokens 19, 36, 33 and 16, 25, 57; 1,024 34, 44, 63 and 19, 25, 79.
constexpr int kTileFrom = 40960;
bool by_tiles(const umem_adapter_desc& ad, int T) { return static_cast<int64_t>(T) * ad.rank >= kTileFrom; }

// Pieces of d_in: the widest that make 512 workgroups (two for each CU; 1,024 were no faster), as wider ones
// leave fewer partial sums.  nb: 16-byte pieces of x to a thread.  8 of bf16 take 66 KiB of LDS, two workgroups
// to a CU; of fp32 (three parts) 99 KiB, one: 4,096 tokens by 2,048 then take 16.5 us, with 4 13.6.
// Workgroups walk several of the widest pieces, adding up their sums, where that leaves this many: the sums are then
// of no more tiles than that, or one for each token, whatever d_in is.  A sum for every piece was as many bytes as
// fp32 x itself at rank 128, and 2 GB of scratch for 8,192 tokens by 65,536 (1,687 us; 67 MB and 1,467 so).  65,536 fp32
// tokens by 2,048, rank 64: 494 us and 268 MB, 481 and 34 so; with 512 workgroups 500, with 1,024 500, with 4,096
// 489.  (bf16 x has a quarter of the sums: 32,768 tokens by 8,192, rank 128, 488 us, 479 so; 131,072 by 2,048,
// rank 64, 419 us, 424 so.)
constexpr int kLowWorkgroups = 512, kWalkWorkgroups = 2048;
struct Plan {
  int nb, piece, pieces, walk, runs, splits, rank_tiles;       // walk: pieces of a run
};
Plan plan_of(const umem_adapter_desc& ad, int T) {
  Plan p;
  const int tiles = (T + kTile - 1) / kTile;
  const int widest = ad.xtype == UMEM_F32 ? 4 : 8;
  for (p.nb = widest;; p.nb /= 2) {
    p.piece = ad.xtype == UMEM_F32 ? piece_width<float>(p.nb) : piece_width<__bf16>(p.nb);
    p.pieces = (ad.d_in + p.piece - 1) / p.piece;
    if (p.nb == 1 || static_cast<int64_t>(tiles) * p.pieces >= kLowWorkgroups) break;
  }
  p.runs = p.nb == widest ? std::min(p.pieces, std::max(1, kWalkWorkgroups / tiles)) : p.pieces;
  p.walk = (p.pieces + p.runs - 1) / p.runs;
  p.runs = (p.pieces + p.walk - 1) / p.walk;
  p.splits = std::max(1, std::min(512 / tiles, (ad.d_out + 127) / 128));
  p.rank_tiles = (ad.rank + 15) / 16;
  return p;
}

}  // namespace

// The most that T tokens or fewer take: fewer tiles have narrower pieces, which leave more sums of a token (bf16 x of
// 4,096, rank 32: 4,032 tokens 8.3 MB, 4,096 4.2).  So every width that T tokens or fewer take is looked at, at the
// most tokens that take it; runs of pieces have at most kWalkWorkgroups tiles of sums, or one for each token.
size_t adapter_workspace_bytes(const umem_adapter_desc& ad, int T) {
  size_t most = 0;
  while (T > 0 && by_tiles(ad, T)) {
    const Plan p = plan_of(ad, T);
    const size_t sums = std::min(static_cast<size_t>(p.pieces) * T, std::max<size_t>(kWalkWorkgroups * kTile, T));
    most = std::max(most, (sums * p.rank_tiles * 16 * sizeof(float) + 255) / 256 * 256);
    if (p.nb == 1) break;
    T = ((kLowWorkgroups + p.pieces - 1) / p.pieces - 1) * kTile;
  }
  return most;
}

hipError_t launch_adapter_add(const umem_adapter_desc& ad, int T, const void* x, const int32_t* ids,
                              const uint16_t* a, const uint16_t* b, const float* scale, const void* base,
                              void* out, void* ws, hipStream_t s) {
  clear_stale_error();
  AdapterArgs k{x, ids, a, b, scale, base, out, T, ad.n, ad.rank, ad.d_in, ad.d_out, 1, nullptr, 0};
  if (!by_tiles(ad, T)) {
    k.splits = std::max(1, std::min(256 / T, (ad.d_out + kTokenThreads - 1) / kTokenThreads));
    const int rows = (ad.rank + kTokenWaves - 1) / kTokenWaves;
#define UMEM_TOKEN(XT, OT, ROWS) \
  hipLaunchKernelGGL((token_kernel<XT, OT, ROWS>), dim3(T, k.splits), dim3(kTokenThreads), 0, s, k)
#define UMEM_ADAPTER(XT, OT)                   \
  if (rows <= 1) UMEM_TOKEN(XT, OT, 1);        \
  else if (rows <= 2) UMEM_TOKEN(XT, OT, 2);   \
  else if (rows <= 4) UMEM_TOKEN(XT, OT, 4);   \
  else if (rows <= 8) UMEM_TOKEN(XT, OT, 8);   \
  else UMEM_TOKEN(XT, OT, 16);
    if (ad.xtype == UMEM_F32 && ad.otype == UMEM_F32) { UMEM_ADAPTER(float, float) }
    else if (ad.xtype == UMEM_F32) { UMEM_ADAPTER(float, __bf16) }
    else if (ad.otype == UMEM_F32) { UMEM_ADAPTER(__bf16, float) }
    else { UMEM_ADAPTER(__bf16, __bf16) }
#undef UMEM_ADAPTER
#undef UMEM_TOKEN
    return hipGetLastError();
  }
  const Plan p = plan_of(ad, T);
  const int tiles = (T + kTile - 1) / kTile;
  k.splits = p.splits;
  k.low = static_cast<float*>(ws);
  k.runs = p.runs;
  const dim3 grid(tiles, p.runs), block(kThreads);
  const size_t lds = static_cast<size_t>(kTile) * (p.piece + 8) * 2 * (ad.xtype == UMEM_F32 ? 3 : 1);
#define UMEM_LOW(XT, NB, CG, WALK) \
  hipLaunchKernelGGL((low_kernel<XT, NB, CG, WALK>), grid, block, lds, s, k, p.rank_tiles, p.walk)
#define UMEM_LOW_RANK(XT, NB, WALK)                \
  if (ad.rank <= 32) UMEM_LOW(XT, NB, 1, WALK);    \
  else UMEM_LOW(XT, NB, 2, WALK);
#define UMEM_ADAPTER(XT)                                \
  if (p.nb == 4) { UMEM_LOW_RANK(XT, 4, false) }        \
  else if (p.nb == 2) { UMEM_LOW_RANK(XT, 2, false) }   \
  else { UMEM_LOW_RANK(XT, 1, false) }
  if (ad.xtype == UMEM_F32 && p.walk > 1) { UMEM_LOW_RANK(float, 4, true) }
  else if (ad.xtype == UMEM_F32) { UMEM_ADAPTER(float) }
  else if (p.walk > 1) { UMEM_LOW_RANK(__bf16, 8, true) }
  else if (p.nb == 8) { UMEM_LOW_RANK(__bf16, 8, false) }
  else { UMEM_ADAPTER(__bf16) }
#undef UMEM_ADAPTER
#undef UMEM_LOW_RANK
#undef UMEM_LOW
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
#define UMEM_OUT(OT, KT) hipLaunchKernelGGL((out_kernel<OT, KT>), dim3(tiles, p.splits), block, 0, s, k, p.rank_tiles)
#define UMEM_ADAPTER(OT)                    \
  if (ad.rank <= 32) UMEM_OUT(OT, 1);       \
  else if (ad.rank <= 64) UMEM_OUT(OT, 2);  \
  else UMEM_OUT(OT, 4);
  if (ad.otype == UMEM_F32) { UMEM_ADAPTER(float) }
  else { UMEM_ADAPTER(__bf16) }
#undef UMEM_ADAPTER
#undef UMEM_OUT
  return hipGetLastError();
}

}  // namespace umem
