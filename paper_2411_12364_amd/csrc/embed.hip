// Token rows: the lookup of a model's first operator, and its gradient by sorted tokens.
//
//   out[t] = s E[ids[t]],    dE[v] += s sum over t with ids[t] = v of dout[t]
//
// Both move memory and compute next to nothing.  The gradient sorts the (token, place) pairs, so that every row of the
// table is summed by its places in order: no atomics, the same bits each time.  Up to 4,096 places are sorted by one
// workgroup in LDS, up to 32,768 by a launch a pass, as a chain of short launches costs more than what they do (8,192
// places: 11 us in two, 23 by sort.hip's six, 17 by one workgroup with eight places a thread).  A wave takes a run of sorted places
// and 256 columns; a row that begins and ends within its run is written at once, what is left at
// the run's two ends goes to scratch, and a second kernel adds the pieces of rows that pass from run to run.
#include <algorithm>

#include "umem_internal.h"

namespace umem {
namespace {

constexpr int kThreads = 256;
constexpr uint32_t kNone = 0xffffffffu;         // the key of a place without a row

typedef float f32x4 __attribute__((ext_vector_type(4)));

// Four elements at any element's alignment (global loads and stores of 8 and 16 bytes need none).
template <typename T>
struct Four {
  typedef T type __attribute__((ext_vector_type(4), aligned(sizeof(T))));
};

template <typename T>
__device__ __forceinline__ f32x4 load4(const T* p) {
  const typename Four<T>::type v = *reinterpret_cast<const typename Four<T>::type*>(p);
  return f32x4{static_cast<float>(v.x), static_cast<float>(v.y), static_cast<float>(v.z), static_cast<float>(v.w)};
}
template <typename T>
__device__ __forceinline__ void store4(T* p, f32x4 v) {
  const typename Four<T>::type o = {static_cast<T>(v.x), static_cast<T>(v.y), static_cast<T>(v.z), static_cast<T>(v.w)};
  *reinterpret_cast<typename Four<T>::type*>(p) = o;
}
// The first n < 4 elements.
template <typename T>
__device__ __forceinline__ f32x4 load_part(const T* p, int n) {
  f32x4 v = {0.f, 0.f, 0.f, 0.f};
  if (n > 0) v.x = static_cast<float>(p[0]);
  if (n > 1) v.y = static_cast<float>(p[1]);
  if (n > 2) v.z = static_cast<float>(p[2]);
  return v;
}
template <typename T>
__device__ __forceinline__ void store_part(T* p, f32x4 v, int n) {
  if (n > 0) p[0] = static_cast<T>(v.x);
  if (n > 1) p[1] = static_cast<T>(v.y);
  if (n > 2) p[2] = static_cast<T>(v.z);
}

// A wave copies kCols columns of one token, four or eight of them a lane.  Bounded by HBM: 16,381 rows of 1,023 fp32 22.5
// us, 4.7 TB/s (a large copy 5.0); 32 rows of 2,048 bf16 2.3 us, the launch and two loads in turn.
constexpr int kCols = 512;

template <typename WT, typename OT>
__global__ __launch_bounds__(kThreads) void embed_kernel(const WT* __restrict__ table, const int32_t* __restrict__ ids,
                                                         OT* __restrict__ out, int T, int vocab, int d, int slabs,
                                                         float scale) {
  const int lane = threadIdx.x & (kWave - 1);
  const int64_t item = static_cast<int64_t>(blockIdx.x) * (kThreads / kWave) + threadIdx.x / kWave;
  const int t = __builtin_amdgcn_readfirstlane(static_cast<int>(item / slabs));
  const int c0 = __builtin_amdgcn_readfirstlane(static_cast<int>(item % slabs)) * kCols;
  if (t >= T) return;
  const int32_t id = ids[t];
  const bool on = static_cast<uint32_t>(id) < static_cast<uint32_t>(vocab);
  const WT* row = table + static_cast<int64_t>(on ? id : 0) * d;
  OT* to = out + static_cast<int64_t>(t) * d;
#pragma unroll
  for (int i = 0; i < kCols / (4 * kWave); ++i) {
    const int c = c0 + (i * kWave + lane) * 4;
    if (c + 4 <= d) {
      const f32x4 v = on ? load4(row + c) * scale : f32x4{0.f, 0.f, 0.f, 0.f};
      store4(to + c, v);
    } else if (c < d) {
      const f32x4 v = on ? load_part(row + c, d - c) * scale : f32x4{0.f, 0.f, 0.f, 0.f};
      store_part(to + c, v, d - c);
    }
  }
}

// The sort's keys, and the counts of their first digit by tiles.
__global__ __launch_bounds__(kSortThreads) void embed_keys_kernel(const int32_t* __restrict__ ids, int T, int vocab,
                                                                  uint32_t* __restrict__ keys, int dbits, int tile,
                                                                  int tiles, uint32_t* __restrict__ hist) {
  __shared__ uint32_t count[1 << kSortMaxDigitBits];
  const int nd = 1 << dbits;
  for (int i = threadIdx.x; i < nd; i += kSortThreads) count[i] = 0;
  __syncthreads();
  const int first = blockIdx.x * tile, last = min(T, first + tile);
  for (int t = first + threadIdx.x; t < last; t += kSortThreads) {
    const uint32_t id = static_cast<uint32_t>(ids[t]);
    const bool on = id < static_cast<uint32_t>(vocab);
    keys[t] = on ? id : kNone;
    if (on) atomicAdd(&count[id & (nd - 1)], 1u);
  }
  __syncthreads();
  for (int i = threadIdx.x; i < nd; i += kSortThreads) hist[static_cast<size_t>(i) * tiles + blockIdx.x] = count[i];
}

// Rows by their order: a sorted place begins a row where its key is another than the one before.
constexpr int kRankTile = 1024;

__device__ __forceinline__ bool begins(const uint2* pairs, int e) { return e == 0 || pairs[e - 1].x != pairs[e].x; }

__global__ __launch_bounds__(kThreads) void embed_count_kernel(const uint2* __restrict__ pairs,
                                                               const uint32_t* __restrict__ n_pairs,
                                                               uint32_t* __restrict__ starts) {
  __shared__ uint32_t total;
  if (threadIdx.x == 0) total = 0;
  __syncthreads();
  const int n = static_cast<int>(*n_pairs), first = blockIdx.x * kRankTile;
  uint32_t mine = 0;
  for (int e = first + threadIdx.x; e < min(n, first + kRankTile); e += kThreads) mine += begins(pairs, e);
  if (mine) atomicAdd(&total, mine);
  __syncthreads();
  if (threadIdx.x == 0) starts[blockIdx.x] = total;
}

// place[e]: the number of the row that sorted place e belongs to; rows, n_rows as the call returns them.
__global__ __launch_bounds__(kThreads) void embed_rank_kernel(const uint2* __restrict__ pairs,
                                                              const uint32_t* __restrict__ n_pairs,
                                                              const uint32_t* __restrict__ starts,
                                                              uint32_t* __restrict__ place, int32_t* __restrict__ rows,
                                                              int32_t* __restrict__ n_rows) {
  __shared__ uint32_t wave_sum[kThreads / kWave];
  __shared__ uint32_t before;
  const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
  if (threadIdx.x == 0) before = 0;
  __syncthreads();
  uint32_t mine = 0;
  for (int i = threadIdx.x; i < static_cast<int>(blockIdx.x); i += kThreads) mine += starts[i];
  if (mine) atomicAdd(&before, mine);
  __syncthreads();
  uint32_t run = before;
  const int n = static_cast<int>(*n_pairs), first = blockIdx.x * kRankTile, last = min(n, first + kRankTile);
  for (int e0 = first; e0 < first + kRankTile; e0 += kThreads) {
    const int e = e0 + threadIdx.x;
    const bool on = e < last && begins(pairs, e);
    const uint64_t ballot = __ballot(on);
    if (lane == 0) wave_sum[wave] = static_cast<uint32_t>(__popcll(ballot));
    __syncthreads();
    uint32_t at = run;
#pragma unroll
    for (int w = 0; w < kThreads / kWave; ++w) {
      at += w < wave ? wave_sum[w] : 0u;
      run += wave_sum[w];
    }
    at += static_cast<uint32_t>(__popcll(ballot & lanemask_lt())) + (on ? 1u : 0u);     // rows begun up to e
    if (e < last) place[e] = at - 1;
    if (on) rows[at - 1] = static_cast<int32_t>(pairs[e].x);
    __syncthreads();
  }
  if (blockIdx.x == gridDim.x - 1 && threadIdx.x == 0) *n_rows = static_cast<int32_t>(run);
}

// The lanes that have this lane's 8-bit digit.
__device__ __forceinline__ uint64_t same_digit(uint32_t digit) {
  uint64_t peers = ~0ull;
#pragma unroll
  for (int b = 0; b < 8; ++b) {
    const bool one = digit >> b & 1u;
    const uint64_t ones = __ballot(one);
    peers &= one ? ones : ~ones;
  }
  return peers;
}

// Up to kSmallWaves * 64 * STEPS places by one workgroup: a stable radix sort by 8 bits of the key a pass, of words that
// hold key and place.  A wave ranks its own places, 64 a step, by its running counts of the digit and the lanes
// below with the same one; the words then change places in LDS.  Places without a row have the key `vocab`, past all
// rows.  With place the rows' order as well: place, rows and n_rows as embed_rank_kernel writes them.
constexpr int kSmallWaves = 16, kSmallThreads = kSmallWaves * kWave, kSmallSteps = 4;
constexpr int kSmallPlaces = kSmallThreads * kSmallSteps;

template <int STEPS>
__global__ __launch_bounds__(kSmallThreads) void embed_sort_kernel(const int32_t* __restrict__ ids, int T, int vocab,
                                                                   int place_bits, int passes, uint2* __restrict__ pairs,
                                                                   uint32_t* __restrict__ n_pairs,
                                                                   uint32_t* __restrict__ place, int32_t* __restrict__ rows,
                                                                   int32_t* __restrict__ n_rows) {
  constexpr int kPlaces = kSmallThreads * STEPS;
  __shared__ uint32_t words[kPlaces];
  __shared__ uint16_t count[kSmallWaves][256];
  __shared__ uint32_t wave_sum[kSmallWaves], total;
  const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = tid / kWave;
  const int first = wave * STEPS * kWave + lane;
  uint32_t w[STEPS];
#pragma unroll
  for (int q = 0; q < STEPS; ++q) {
    const int t = first + q * kWave;
    const uint32_t id = t < T ? static_cast<uint32_t>(ids[t]) : 0u;
    const uint32_t key = min(id, static_cast<uint32_t>(vocab));
    w[q] = t < T ? key << place_bits | static_cast<uint32_t>(t) : 0xffffffffu;
  }
  if (tid == 0) total = static_cast<uint32_t>(T);
  for (int pass = 0; pass < passes; ++pass) {
    const int shift = place_bits + 8 * pass;
#pragma unroll
    for (int i = 0; i < 256 / kWave; ++i) count[wave][i * kWave + lane] = 0;
    wave_lds_order();
    uint16_t rank[STEPS];
#pragma unroll
    for (int q = 0; q < STEPS; ++q) {
      const uint32_t digit = w[q] >> shift & 255u;
      const uint64_t peers = same_digit(digit);
      const uint32_t below = static_cast<uint32_t>(__popcll(peers & lanemask_lt()));
      const uint32_t have = count[wave][digit];
      rank[q] = static_cast<uint16_t>(have + below);
      wave_lds_order();
      if (below == 0) count[wave][digit] = static_cast<uint16_t>(have + __popcll(peers));
      wave_lds_order();
    }
    __syncthreads();
    // where each wave's first place of each digit goes: the digits before, then the waves before
    uint32_t all = 0;
    if (tid < 256) {
#pragma unroll
      for (int v = 0; v < kSmallWaves; ++v) all += count[v][tid];
    }
    const uint32_t incl = static_cast<uint32_t>(wave_inclusive_scan(static_cast<int>(all)));
    if (lane == kWave - 1) wave_sum[wave] = incl;
    __syncthreads();
    if (tid < 256) {
      uint32_t at = incl - all;
#pragma unroll
      for (int v = 0; v < 256 / kWave; ++v) at += v < wave ? wave_sum[v] : 0u;
#pragma unroll
      for (int v = 0; v < kSmallWaves; ++v) {
        const uint32_t c = count[v][tid];
        count[v][tid] = static_cast<uint16_t>(at);          // below 2^16: the places are at most 2^15
        at += c;
      }
    }
    __syncthreads();
#pragma unroll
    for (int q = 0; q < STEPS; ++q) words[count[wave][w[q] >> shift & 255u] + rank[q]] = w[q];
    __syncthreads();
#pragma unroll
    for (int q = 0; q < STEPS; ++q) w[q] = words[first + q * kWave];
  }
  // (a wave's words are its own from here on but for the one before them)
  const uint32_t mask = (1u << place_bits) - 1u;
  uint32_t starts = 0;
#pragma unroll
  for (int q = 0; q < STEPS; ++q) {
    const int e = first + q * kWave;
    const uint32_t key = w[q] >> place_bits;
    const uint32_t left = e > 0 ? words[e - 1] >> place_bits : 0xffffffffu;
    const bool row = key < static_cast<uint32_t>(vocab);
    if (row) pairs[e] = make_uint2(key, w[q] & mask);
    if (!row && e < T && (e == 0 || left < static_cast<uint32_t>(vocab))) total = static_cast<uint32_t>(e);
    starts += static_cast<uint32_t>(__popcll(__ballot(row && left != key)));
  }
  if (lane == 0) wave_sum[wave] = starts;
  __syncthreads();
  if (tid == 0) *n_pairs = total;
  if (place == nullptr) return;
  uint32_t run = 0, rows_all = 0;
#pragma unroll
  for (int v = 0; v < kSmallWaves; ++v) {
    run += v < wave ? wave_sum[v] : 0u;
    rows_all += wave_sum[v];
  }
  if (tid == 0) *n_rows = static_cast<int32_t>(rows_all);
#pragma unroll
  for (int q = 0; q < STEPS; ++q) {
    const int e = first + q * kWave;
    const uint32_t key = w[q] >> place_bits;
    const bool row = key < static_cast<uint32_t>(vocab), begin = row && (e == 0 || words[e - 1] >> place_bits != key);
    const uint64_t ballot = __ballot(begin);
    const uint32_t at = run + static_cast<uint32_t>(__popcll(ballot & (lanemask_lt() << 1 | 1ull))) - 1u;   // rows begun up to e
    if (row) place[e] = at;
    if (begin) rows[at] = static_cast<int32_t>(key);
    run += static_cast<uint32_t>(__popcll(ballot));
  }
}

// One pass over up to kPassPlaces places, a tile of 512 a workgroup: it counts all digits itself, those of the tiles before
// its own apart, so that no other kernel stands between (8,192 places 5.3 us a pass, 20,000 8.4, where sort.hip's three
// kernels a pass take 13), ranks its tile's places, one a lane, and writes their words to their new places.  The first
// pass makes the words from ids, the last writes pairs.
constexpr int kPassThreads = 512, kPassWaves = kPassThreads / kWave, kPassPlaces = 32 << 10;

__global__ __launch_bounds__(kPassThreads) void embed_pass_kernel(const int32_t* __restrict__ ids,
                                                                  const uint32_t* __restrict__ in, int T, int vocab,
                                                                  int place_bits, int shift, bool last,
                                                                  uint32_t* __restrict__ out, uint2* __restrict__ pairs,
                                                                  uint32_t* __restrict__ n_pairs) {
  // (16 copies of each count: tokens' high digits are few, and lanes that add to one word wait for each other)
  constexpr int kCopies = 16;
  __shared__ uint32_t before[256][kCopies], after[256][kCopies], base[256];
  __shared__ uint16_t count[kPassWaves][256];
  __shared__ uint32_t wave_sum[4], rowless;
  const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = tid / kWave;
  const int tile0 = blockIdx.x * kPassThreads;
#pragma unroll
  for (int i = 0; i < 256 * kCopies / kPassThreads; ++i)
    (&before[0][0])[i * kPassThreads + tid] = (&after[0][0])[i * kPassThreads + tid] = 0;
  if (tid == 0) rowless = 0;
#pragma unroll
  for (int i = 0; i < 256 / kWave; ++i) count[wave][i * kWave + lane] = 0;
  __syncthreads();
  typedef uint32_t four __attribute__((ext_vector_type(4), aligned(4)));
  const uint32_t* from = in != nullptr ? in : reinterpret_cast<const uint32_t*>(ids);
  const auto word = [&](uint32_t v, int t) {
    return in != nullptr ? v : min(v, static_cast<uint32_t>(vocab)) << place_bits | static_cast<uint32_t>(t);
  };
  uint32_t none = 0;
  const auto add = [&](uint32_t v, int t) {
    const uint32_t w = word(v, t);
    atomicAdd((t < tile0 ? before : after)[w >> shift & 255u] + lane % kCopies, 1u);
    none += (w >> place_bits) >= static_cast<uint32_t>(vocab);
  };
  constexpr int kFours = 4;               // loads under way
  for (int t0 = tid * 4; t0 < T; t0 += kFours * 4 * kPassThreads) {
    four v[kFours];
#pragma unroll
    for (int i = 0; i < kFours; ++i)
      v[i] = *reinterpret_cast<const four*>(from + max(min(t0 + i * 4 * kPassThreads, T - 4), 0));
#pragma unroll
    for (int i = 0; i < kFours; ++i) {
      const int t = t0 + i * 4 * kPassThreads;
      if (t + 4 <= T) {
#pragma unroll
        for (int j = 0; j < 4; ++j) add(v[i][j], t + j);
      } else {
        for (int e = t; e < T; ++e) add(from[e], e);
      }
    }
  }
  const int t = tile0 + tid;
  const uint32_t w = t < T ? word(from[t], t) : 0xffffffffu, digit = w >> shift & 255u;
  const uint64_t peers = same_digit(digit) & __ballot(t < T);
  const uint32_t rank = static_cast<uint32_t>(__popcll(peers & lanemask_lt()));
  if (t < T && rank == 0) count[wave][digit] = static_cast<uint16_t>(__popcll(peers));
  if (last && none) atomicAdd(&rowless, none);
  __syncthreads();
  uint32_t all = 0, incl = 0, ahead = 0;
  if (tid < 256) {
#pragma unroll
    for (int i = 0; i < kCopies; ++i) {
      const int c = (i + tid) % kCopies;
      ahead += before[tid][c];
      all += after[tid][c];
    }
    all += ahead;
    incl = static_cast<uint32_t>(wave_inclusive_scan(static_cast<int>(all)));
    if (lane == kWave - 1) wave_sum[wave] = incl;
  }
  __syncthreads();
  if (tid < 256) {
    uint32_t at = incl - all + ahead;
#pragma unroll
    for (int v = 0; v < 4; ++v) at += v < wave ? wave_sum[v] : 0u;
    base[tid] = at;
    uint32_t run = 0;
#pragma unroll
    for (int v = 0; v < kPassWaves; ++v) {
      const uint32_t c = count[v][tid];
      count[v][tid] = static_cast<uint16_t>(run);
      run += c;
    }
  }
  __syncthreads();
  if (last && blockIdx.x == 0 && tid == 0) *n_pairs = static_cast<uint32_t>(T) - rowless;
  if (t >= T) return;
  const uint32_t to = base[digit] + count[wave][digit] + rank, key = w >> place_bits;
  if (!last) out[to] = w;
  else if (key < static_cast<uint32_t>(vocab)) pairs[to] = make_uint2(key, w & ((1u << place_bits) - 1u));
}

// Where a finished row goes: added to the dense table, or written to its compact row.
template <bool ROWS>
__device__ __forceinline__ void put_row(float* out, int64_t row, int d, int c, f32x4 v, float scale) {
  float* p = out + row * d + c;
  if (c + 4 <= d) {
    f32x4 o = v * scale;
    if constexpr (!ROWS) {
      const f32x4 h = load4(p);
#pragma unroll
      for (int i = 0; i < 4; ++i) o[i] = fmaf(v[i], scale, h[i]);
    }
    store4(p, o);
  } else {
    for (int i = 0; i < d - c; ++i) p[i] = ROWS ? v[i] * scale : fmaf(v[i], scale, p[i]);
  }
}

constexpr int kSlab = 4 * kWave;                // columns of a wave
constexpr int kAhead = 8;                       // rows a wave has in flight

// Sums of the runs of `run` sorted places.  edge: fp32 [runs][2][d]: what a run adds to the row that the run
// before it left open, and what it leaves open itself.  Bounded by HBM: 8,192 places of 2,048 bf16 20 us, 4.5 TB/s of 92 MB.
template <typename GT, bool ROWS>
__global__ __launch_bounds__(kThreads) void embed_sum_kernel(const uint2* __restrict__ pairs,
                                                             const uint32_t* __restrict__ n_pairs,
                                                             const uint32_t* __restrict__ place,
                                                             const GT* __restrict__ dout, float* __restrict__ out,
                                                             float* __restrict__ edge, int run, int slabs, int d,
                                                             float scale) {
  const int lane = threadIdx.x & (kWave - 1);
  const int64_t item = static_cast<int64_t>(blockIdx.x) * (kThreads / kWave) + threadIdx.x / kWave;
  const int r = __builtin_amdgcn_readfirstlane(static_cast<int>(item / slabs));
  const int c = __builtin_amdgcn_readfirstlane(static_cast<int>(item % slabs)) * kSlab + lane * 4;
  const int n = static_cast<int>(*n_pairs);
  const int first = r * run, last = min(n, first + run);
  if (first >= n) return;
  const bool whole = c + 4 <= d, part = !whole && c < d;
  uint32_t key = pairs[first].x;
  bool open = first > 0 && pairs[first - 1].x == key;       // the row began before this run
  f32x4 sum = {0.f, 0.f, 0.f, 0.f};
  const auto leave = [&](int64_t at) {
    float* p = edge + at * d + c;
    if (whole) store4(p, sum);
    else if (part) store_part(p, sum, d - c);
  };
  for (int e0 = first; e0 < last; e0 += kAhead) {
    f32x4 v[kAhead];
    uint2 pr[kAhead];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) pr[i] = pairs[min(e0 + i, last - 1)];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      const GT* p = dout + static_cast<int64_t>(pr[i].y) * d + c;
      v[i] = whole ? load4(p) : f32x4{0.f, 0.f, 0.f, 0.f};
      if (part) v[i] = load_part(p, d - c);
    }
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      if (e0 + i >= last) break;
      if (pr[i].x != key) {
        if (open) leave(2 * static_cast<int64_t>(r));
        else if (c < d) put_row<ROWS>(out, ROWS ? static_cast<int64_t>(place[e0 + i - 1]) : key, d, c, sum, scale);
        open = false;
        key = pr[i].x;
        sum = f32x4{0.f, 0.f, 0.f, 0.f};
      }
      sum += v[i];
    }
  }
  if (open) leave(2 * static_cast<int64_t>(r));
  else if (last < n && pairs[last].x == key) leave(2 * static_cast<int64_t>(r) + 1);
  else if (c < d) put_row<ROWS>(out, ROWS ? static_cast<int64_t>(place[last - 1]) : key, d, c, sum, scale);
}

// Rows that pass from run to run: the workgroup of the run that a row begins in adds what the following runs hold of
// it, each wave a quarter of them.
template <bool ROWS>
__global__ __launch_bounds__(kThreads) void embed_join_kernel(const uint2* __restrict__ pairs,
                                                              const uint32_t* __restrict__ n_pairs,
                                                              const uint32_t* __restrict__ place,
                                                              float* __restrict__ out, const float* __restrict__ edge,
                                                              int run, int d, float scale) {
  constexpr int kWaves = kThreads / kWave;
  __shared__ f32x4 part[kWaves][kWave];
  const int lane = threadIdx.x & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int r = blockIdx.x, c = blockIdx.y * kSlab + lane * 4;
  const int n = static_cast<int>(*n_pairs);
  const int first = r * run, last = first + run;
  if (last >= n) return;                                    // nothing follows
  const uint32_t key = pairs[last - 1].x, before = first > 0 ? pairs[first - 1].x : ~key;
  if (pairs[last].x != key || before == key) return;        // (the whole workgroup)
  // the runs after this one that hold more of the row: all but the last of them end within it
  const int runs = (n + run - 1) / run;
  int more = 0;
  for (int r0 = r + 1; r0 < runs; r0 += kWave) {
    const int q = r0 + lane;
    const bool ends = q >= runs - 1 || pairs[static_cast<int64_t>(q + 1) * run].x != key;
    const uint64_t ballot = __ballot(ends);
    if (ballot != 0) {
      more += __ffsll(static_cast<unsigned long long>(ballot));
      break;
    }
    more += kWave;
  }
  const bool whole = c + 4 <= d;
  const float* p = edge + 2 * static_cast<int64_t>(r) * d + c;
  const auto get = [&](const float* q) { return whole ? load4(q) : load_part(q, d - c); };
  f32x4 sum = {0.f, 0.f, 0.f, 0.f};
  const int share = (more + kWaves - 1) / kWaves, end = min(more, (wave + 1) * share);
  if (c < d) {
    if (wave == 0) sum = get(p + d);
#pragma unroll 8
    for (int i = wave * share + 1; i <= end; ++i) sum += get(p + 2 * static_cast<int64_t>(i) * d);
  }
  part[wave][lane] = sum;
  __syncthreads();
  if (wave != 0 || c >= d) return;
#pragma unroll
  for (int w = 1; w < kWaves; ++w) sum += part[w][lane];
  put_row<ROWS>(out, ROWS ? static_cast<int64_t>(place[last - 1]) : key, d, c, sum, scale);
}

// Sorted places of a run: 16, so that there are many runs, and from 2^16 places on as many as give 4,096 runs; of up
// to 2,048 places 8, which a wave has in flight at once.
constexpr int kShortPlaces = 2048;
int run_length(int T) { return T <= kShortPlaces ? kAhead : std::max(16, (T + 4095) / 4096); }
int most_runs(int T) { return (T + run_length(T) - 1) / run_length(T); }
// The bits of the numbers below `vocab`.
int key_bits(int64_t vocab) {
  int bits = 1;
  while (bits < 32 && (INT64_C(1) << bits) < vocab) ++bits;
  return bits;
}
size_t up256(size_t x) { return (x + 255) & ~static_cast<size_t>(255); }

template <typename GT, bool ROWS>
hipError_t backward(const umem_embed_desc& ed, int T, const int32_t* ids, const GT* dout, float* out, int32_t* rows,
                    int32_t* n_rows, void* ws, hipStream_t s) {
  char* base = static_cast<char*>(ws);
  float* edge = reinterpret_cast<float*>(base + up256(sort_workspace_bytes(T)));
  uint32_t* starts = reinterpret_cast<uint32_t*>(reinterpret_cast<char*>(edge) +
                                                 up256(static_cast<size_t>(most_runs(T)) * 2 * ed.d * sizeof(float)));
  const SortPlan p = sort_plan(T, key_bits(ed.vocab), base);
  const int place_bits = key_bits(T), word_bits = key_bits(ed.vocab + INT64_C(1));
  uint2* sorted = p.a;
  uint32_t* place = reinterpret_cast<uint32_t*>(p.b);
  const int passes = (word_bits + 7) / 8;
  const bool packed = place_bits + word_bits <= 32;
  bool ranked = false;
  if (T <= kSmallPlaces && packed) {
    const auto sort = T <= kSmallThreads ? embed_sort_kernel<1> : embed_sort_kernel<kSmallSteps>;
    hipLaunchKernelGGL(sort, dim3(1), dim3(kSmallThreads), 0, s, ids, T, ed.vocab, place_bits, passes, sorted, p.n,
                       ROWS ? place : nullptr, rows, n_rows);
    ranked = true;
  } else if (T <= kPassPlaces && packed) {
    // the words change between the halves of the other array of pairs
    uint32_t *in = nullptr, *out = reinterpret_cast<uint32_t*>(p.b), *next = out + T;
    for (int pass = 0; pass < passes; ++pass) {
      hipLaunchKernelGGL(embed_pass_kernel, dim3((T + kPassThreads - 1) / kPassThreads), dim3(kPassThreads), 0, s, ids, in, T,
                         ed.vocab, place_bits, place_bits + 8 * pass, pass + 1 == passes, out, sorted, p.n);
      in = out;
      std::swap(out, next);
    }
  } else {
    hipLaunchKernelGGL(embed_keys_kernel, dim3(p.tiles), dim3(kSortThreads), 0, s, ids, T, ed.vocab, p.keys, p.dbits, p.tile,
                       p.tiles, p.hist);
    uint2* dead;
    const hipError_t e = sort_run(p, kNone, true, s, &sorted, &dead);
    if (e != hipSuccess) return e;
    place = reinterpret_cast<uint32_t*>(dead);
  }
  if (ROWS && !ranked) {
    const int tiles = (T + kRankTile - 1) / kRankTile;
    hipLaunchKernelGGL(embed_count_kernel, dim3(tiles), dim3(kThreads), 0, s, sorted, p.n, starts);
    hipLaunchKernelGGL(embed_rank_kernel, dim3(tiles), dim3(kThreads), 0, s, sorted, p.n, starts, place, rows, n_rows);
  }
  const int slabs = (ed.d + kSlab - 1) / kSlab, run = run_length(T);
  const int64_t items = static_cast<int64_t>(most_runs(T)) * slabs;
  const dim3 grid(static_cast<unsigned>((items + 3) / 4));
  hipLaunchKernelGGL((embed_sum_kernel<GT, ROWS>), grid, dim3(kThreads), 0, s, sorted, p.n, place, dout, out, edge, run,
                     slabs, ed.d, ed.scale);
  if (most_runs(T) > 1)
    hipLaunchKernelGGL((embed_join_kernel<ROWS>), dim3(most_runs(T), slabs), dim3(kThreads), 0, s, sorted, p.n, place, out,
                       edge, run, ed.d, ed.scale);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_embed(const umem_embed_desc& ed, int T, const void* table, const int32_t* ids, void* out,
                        hipStream_t s) {
  clear_stale_error();
  const int slabs = (ed.d + kCols - 1) / kCols;
  const int64_t items = static_cast<int64_t>(T) * slabs;
  const dim3 grid(static_cast<unsigned>((items + 3) / 4));
  const auto go = [&](auto* w, auto* o) {
    hipLaunchKernelGGL(embed_kernel, grid, dim3(kThreads), 0, s, w, ids, o, T, ed.vocab, ed.d, slabs, ed.scale);
  };
  const float* wf = static_cast<const float*>(table);
  const __bf16* wb = static_cast<const __bf16*>(table);
  if (ed.wtype == UMEM_F32) {
    if (ed.otype == UMEM_F32) go(wf, static_cast<float*>(out));
    else go(wf, static_cast<__bf16*>(out));
  } else {
    if (ed.otype == UMEM_F32) go(wb, static_cast<float*>(out));
    else go(wb, static_cast<__bf16*>(out));
  }
  return hipGetLastError();
}

size_t embed_backward_workspace_bytes(const umem_embed_desc& ed, int T) {
  if (T == 0) return 0;
  // (as many runs as any number of tokens up to T has: 4,096 from 2^16 - 15 of them on)
  const int runs = T > (1 << 16) - 16 ? 4096 : std::max(most_runs(T), most_runs(std::min(T, kShortPlaces)));
  return up256(sort_workspace_bytes(T)) + up256(static_cast<size_t>(runs) * 2 * ed.d * sizeof(float)) +
         up256(static_cast<size_t>((T + kRankTile - 1) / kRankTile) * sizeof(uint32_t));
}

hipError_t launch_embed_backward(const umem_embed_desc& ed, int T, const int32_t* ids, const void* dout, float* out,
                                 int32_t* rows, int32_t* n_rows, void* ws, hipStream_t s) {
  clear_stale_error();
  if (ed.otype == UMEM_F32) {
    const float* g = static_cast<const float*>(dout);
    return rows ? backward<float, true>(ed, T, ids, g, out, rows, n_rows, ws, s)
                : backward<float, false>(ed, T, ids, g, out, rows, n_rows, ws, s);
  }
  const __bf16* g = static_cast<const __bf16*>(dout);
  return rows ? backward<__bf16, true>(ed, T, ids, g, out, rows, n_rows, ws, s)
              : backward<__bf16, false>(ed, T, ids, g, out, rows, n_rows, ws, s);
}

}  // namespace umem
