// Token rows: the lookup of a model's first operator, and its gradient by sorted tokens.
//
//   out[t] = s E[ids[t]],    dE[v] += s sum over t with ids[t] = v of dout[t]
//
// Both move memory and compute next to nothing.  The gradient sorts the (token, place) pairs, so that every row of the
// table is summed by its places in order: no atomics, the same bits each time.  A wave takes a run of sorted places
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

// A wave copies kCols columns of one token, four or eight of them a lane.
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
constexpr int kRankTile = 4096;

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
// before it left open, and what it leaves open itself.
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

// Rows that pass from run to run: the wave of the run that a row begins in adds what the following runs hold of it.
template <bool ROWS>
__global__ __launch_bounds__(kThreads) void embed_join_kernel(const uint2* __restrict__ pairs,
                                                              const uint32_t* __restrict__ n_pairs,
                                                              const uint32_t* __restrict__ place,
                                                              float* __restrict__ out, const float* __restrict__ edge,
                                                              int run, int slabs, int d, float scale) {
  const int lane = threadIdx.x & (kWave - 1);
  const int64_t item = static_cast<int64_t>(blockIdx.x) * (kThreads / kWave) + threadIdx.x / kWave;
  const int r = __builtin_amdgcn_readfirstlane(static_cast<int>(item / slabs));
  const int c = __builtin_amdgcn_readfirstlane(static_cast<int>(item % slabs)) * kSlab + lane * 4;
  const int n = static_cast<int>(*n_pairs);
  const int first = r * run, last = first + run;
  if (last >= n) return;                                    // nothing follows
  const uint32_t key = pairs[last - 1].x;
  if (pairs[last].x != key || (first > 0 && pairs[first - 1].x == key)) return;
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
  if (c >= d) return;
  const bool whole = c + 4 <= d;
  const float* p = edge + 2 * static_cast<int64_t>(r) * d + c;
  const auto get = [&](const float* q) { return whole ? load4(q) : load_part(q, d - c); };
  f32x4 sum = get(p + d);
#pragma unroll 8
  for (int i = 1; i <= more; ++i) sum += get(p + 2 * static_cast<int64_t>(i) * d);
  put_row<ROWS>(out, ROWS ? static_cast<int64_t>(place[last - 1]) : key, d, c, sum, scale);
}

// Sorted places of a run: 16, so that there are many runs, and from 2^16 places on as many as give 4,096 runs.
int run_length(int T) { return std::max(16, (T + 4095) / 4096); }
int most_runs(int T) { return (T + run_length(T) - 1) / run_length(T); }
int key_bits(int vocab) {
  int bits = 1;
  while (bits < 31 && (INT64_C(1) << bits) < vocab) ++bits;
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
  hipLaunchKernelGGL(embed_keys_kernel, dim3(p.tiles), dim3(kSortThreads), 0, s, ids, T, ed.vocab, p.keys, p.dbits, p.tile,
                     p.tiles, p.hist);
  uint2 *sorted, *dead;
  const hipError_t e = sort_run(p, kNone, true, s, &sorted, &dead);
  if (e != hipSuccess) return e;
  uint32_t* place = reinterpret_cast<uint32_t*>(dead);
  if (ROWS) {
    const int tiles = (T + kRankTile - 1) / kRankTile;
    hipLaunchKernelGGL(embed_count_kernel, dim3(tiles), dim3(kThreads), 0, s, sorted, p.n, starts);
    hipLaunchKernelGGL(embed_rank_kernel, dim3(tiles), dim3(kThreads), 0, s, sorted, p.n, starts, place, rows, n_rows);
  }
  const int slabs = (ed.d + kSlab - 1) / kSlab, run = run_length(T);
  const int64_t items = static_cast<int64_t>(most_runs(T)) * slabs;
  const dim3 grid(static_cast<unsigned>((items + 3) / 4));
  hipLaunchKernelGGL((embed_sum_kernel<GT, ROWS>), grid, dim3(kThreads), 0, s, sorted, p.n, place, dout, out, edge, run,
                     slabs, ed.d, ed.scale);
  hipLaunchKernelGGL((embed_join_kernel<ROWS>), grid, dim3(kThreads), 0, s, sorted, p.n, place, out, edge, run, slabs,
                     ed.d, ed.scale);
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
  const int runs = T > (1 << 16) - 16 ? 4096 : most_runs(T);
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
