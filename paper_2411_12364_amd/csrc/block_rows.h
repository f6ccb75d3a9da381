// Rows of a residual stream in the registers of a group of threads (block.hip, block_backward.hip): the
// loads, stores and sums that the norms before and after a block share.  Not part of the public ABI.
#pragma once

#include <algorithm>

#include "umem_internal.h"

namespace umem {

typedef float rf32x4 __attribute__((ext_vector_type(4)));

// Four consecutive elements as they lie in memory.  Rows of an odd width start at any element, so the
// type promises no more than an element's alignment: global loads and stores of 8 and 16 bytes need none.
template <typename T>
struct Quad {
  typedef T type __attribute__((ext_vector_type(4), aligned(sizeof(T))));
};

// A group is 64 threads (a wave; four rows to a workgroup) or a workgroup.  Element (p G + lane) 4 + i of
// a row belongs to v[p][i] of thread `lane`; elements past the row are zeros.
template <int G>
struct Group {
  static constexpr int kThreads = G > 256 ? G : 256;
  static constexpr int kRows = kThreads / G;
  static constexpr int kWaves = G / kWave;
  static __device__ __forceinline__ int lane() { return threadIdx.x % G; }
  static __device__ __forceinline__ int index() { return threadIdx.x / G; }
};

// A row as it lies in memory: half the registers where it is bf16 and waits for its turn.
template <typename T, int PER>
struct RawRow {
  typename Quad<T>::type v[PER];
};
template <int PER>
struct Row {
  rf32x4 v[PER];
};

// How rows end: they fill their group's registers (d = 4 G PER), end between two fours, or within one.
// Loads past a row's fours are sent to its first four and the result dropped, so that only a last, partial
// four takes a branch, of bf16 none.  A branch around every load, and an element by element end in it, cost 900
// rows of 4,092 22 us to leave the block, 14 so; full rows without the selects 4,096 bf16 rows of 2,048 19.0, 20.7
// with them.  bf16 elements taken singly share a register with what the row's other loads write: 8,192 bf16
// rows of 2,047 left the block in 65 us, 50 with the end taken from the row's last four (their backward 100 and
// 69; entry's 66 and 45); fp32 rows are 5 to 15 percent faster with the branch.
enum RowEnd { kFull, kFours, kAny };

// Rows past 8,192, 16 elements to each of 1,024 threads with 128 registers: a group's parameters are read again
// for each row, and few or none of the next row's loads are in flight, or more registers are spilled (1,024 rows of
// 12,288 left the block in 194 us, 89 so, in bf16 135 and 51).  Not all spills are gone: the exit has 6 to 30 of them,
// its backward 42 to 62, entry's backward 0 to 8, and at widths that end within a four 54 to 78, 185 to 220 and up to 99:
// 1,024 fp32 rows of 12,289 leave the block in 154 us (bf16 121), their backward takes 221 (185), entry's 127 (109).
template <int G, int PER>
constexpr bool kWide = G == 1024 && PER == 4;

// Rows of bf16 and the widest, where they end within a four, are masked where they are used, in widen.
template <typename T, int G, int PER, RowEnd END>
constexpr bool kLate = END == kAny && (sizeof(T) == 2 || kWide<G, PER>);

template <int G, int PER, RowEnd END, typename T>
__device__ __forceinline__ RawRow<T, PER> load_raw(const T* row, int lane, int d) {
  RawRow<T, PER> r;
#pragma unroll
  for (int p = 0; p < PER; ++p) {
    const int e = (p * G + lane) * 4;
    if (END == kFull) {
      r.v[p] = *reinterpret_cast<const typename Quad<T>::type*>(row + e);
      continue;
    }
    if (kLate<T, G, PER, END> && d >= 4) {
      // a last, partial four is the row's last four elements
      r.v[p] = *reinterpret_cast<const typename Quad<T>::type*>(row + (e + 4 <= d ? e : e < d ? d - 4 : 0));
      continue;
    }
    r.v[p] = T(0);
    if (END == kFours || d >= 4) {
      const bool in = e + 4 <= d;
      const typename Quad<T>::type x = *reinterpret_cast<const typename Quad<T>::type*>(row + (in ? e : 0));
      r.v[p] = in ? x : r.v[p];
    }
    if (END == kAny && e < d && e + 4 > d) {
      r.v[p].x = row[e];
      if (e + 1 < d) r.v[p].y = row[e + 1];
      if (e + 2 < d) r.v[p].z = row[e + 2];
    }
  }
  return r;
}

template <int G, RowEnd END, typename T, int PER>
__device__ __forceinline__ Row<PER> widen(const RawRow<T, PER>& r, int lane, int d) {
  Row<PER> x;
#pragma unroll
  for (int p = 0; p < PER; ++p) {
    typename Quad<T>::type q = r.v[p];
    if (kLate<T, G, PER, END> && d >= 4) {
      const int e = (p * G + lane) * 4, rest = d & 3;      // 1 to 3 elements, at the end of the last four
      const typename Quad<T>::type last = {rest == 1 ? q.w : rest == 2 ? q.z : q.y,
                                           rest == 1 ? T(0) : rest == 2 ? q.w : q.z, rest == 3 ? q.w : T(0), T(0)};
      q = e + 4 <= d ? q : last;
#pragma unroll
      for (int i = 0; i < 4; ++i) q[i] = e < d ? q[i] : T(0);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) x.v[p][i] = static_cast<float>(q[i]);
  }
  return x;
}

// A vector of parameters [d], or `otherwise` in every element where there is none.
template <int G, int PER, RowEnd END>
__device__ __forceinline__ Row<PER> load_params(const float* p, float otherwise, int lane, int d) {
  if (p != nullptr) return widen<G, END>(load_raw<G, PER, END>(p, lane, d), lane, d);
  Row<PER> r;
#pragma unroll
  for (int q = 0; q < PER; ++q) r.v[q] = otherwise;
  return r;
}

// Parameters of a group's columns, in registers over its rows where there are enough.
template <int G, int PER, RowEnd END>
struct Params {
  static constexpr bool kKept = !kWide<G, PER>;
  const float* p;
  float otherwise;
  Row<PER> kept;
  __device__ __forceinline__ Params(const float* from, float o, int lane, int d) : p(from), otherwise(o) {
    if constexpr (kKept) kept = load_params<G, PER, END>(p, otherwise, lane, d);
  }
  __device__ __forceinline__ Row<PER> row(int lane, int d) const {
    if constexpr (kKept) return kept;
    else return load_params<G, PER, END>(p, otherwise, lane, d);
  }
};

template <int G, RowEnd END, int PER, typename T>
__device__ __forceinline__ void store_row(T* row, const Row<PER>& x, int lane, int d) {
#pragma unroll
  for (int p = 0; p < PER; ++p) {
    const int e = (p * G + lane) * 4;
    const typename Quad<T>::type r = {static_cast<T>(x.v[p].x), static_cast<T>(x.v[p].y), static_cast<T>(x.v[p].z),
                                      static_cast<T>(x.v[p].w)};
    if (END == kFull || e + 4 <= d) {
      *reinterpret_cast<typename Quad<T>::type*>(row + e) = r;
    } else if (END == kAny && e < d) {
      row[e] = r.x;
      if (e + 1 < d) row[e + 1] = r.y;
      if (e + 2 < d) row[e + 2] = r.z;
    }
  }
}

// The sum over a wave in every lane, by data-parallel moves inside the register file (a shuffle
// through LDS costs several times as long, and a row waits for two to five of these sums).
template <int CTRL, int ROWS>
__device__ __forceinline__ float dpp_add(float v) {
  return v + __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(v), CTRL, ROWS, 0xf, false));
}
__device__ __forceinline__ float wave_sum_dpp(float v) {
  v = dpp_add<0xB1, 0xf>(v);       // lane ^ 1
  v = dpp_add<0x4E, 0xf>(v);       // lane ^ 2
  v = dpp_add<0x141, 0xf>(v);      // mirrored in 8 lanes
  v = dpp_add<0x140, 0xf>(v);      // mirrored in 16
  v = dpp_add<0x142, 0xa>(v);      // lane 15 of 16-lane rows 0 and 2 added to rows 1 and 3
  v = dpp_add<0x143, 0xc>(v);      // lane 31 added to rows 2 and 3
  return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(v), 63));
}

// One or two sums over a group: a wave's by wave_sum_dpp, a workgroup's by its waves' sums in LDS, added in wave
// order by every thread (the same bits in all of them).  `turn` picks one of two LDS buffers, so that
// one barrier a sum is enough.
template <int G>
struct GroupSum {
  static constexpr int kWaves = Group<G>::kWaves;
  float (*lds)[kWaves][2];            // [2][kWaves][2]
  int turn;

  __device__ __forceinline__ void sum2(float& a, float& b) {
    a = wave_sum_dpp(a);
    b = wave_sum_dpp(b);
    if constexpr (kWaves > 1) {
      if ((threadIdx.x & (kWave - 1)) == 0) {
        lds[turn][threadIdx.x / kWave][0] = a;
        lds[turn][threadIdx.x / kWave][1] = b;
      }
      __syncthreads();
      a = b = 0.f;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) {
        a += lds[turn][w][0];
        b += lds[turn][w][1];
      }
      turn ^= 1;
    }
  }
  __device__ __forceinline__ float sum(float a) {
    a = wave_sum_dpp(a);
    if constexpr (kWaves > 1) {
      if ((threadIdx.x & (kWave - 1)) == 0) lds[turn][threadIdx.x / kWave][0] = a;
      __syncthreads();
      a = 0.f;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) a += lds[turn][w][0];
      turn ^= 1;
    }
    return a;
  }
};

template <int PER>
__device__ __forceinline__ float add_up(const Row<PER>& x) {
  float s = 0.f;
#pragma unroll
  for (int p = 0; p < PER; ++p) s += (x.v[p].x + x.v[p].y) + (x.v[p].z + x.v[p].w);
  return s;
}
template <int PER>
__device__ __forceinline__ float dot(const Row<PER>& x, const Row<PER>& y) {
  float s = 0.f;
#pragma unroll
  for (int p = 0; p < PER; ++p)
#pragma unroll
    for (int i = 0; i < 4; ++i) s = fmaf(x.v[p][i], y.v[p][i], s);
  return s;
}

template <int G, RowEnd END>
__device__ __forceinline__ bool in_row(int p, int i, int lane, int d) {
  return END == kFull || (p * G + lane) * 4 + (END == kFours ? 0 : i) < d;
}

// x - mean in the row's elements, zeros past it.
template <int G, RowEnd END, int PER>
__device__ __forceinline__ void centre_row(Row<PER>& x, float mean, int lane, int d) {
#pragma unroll
  for (int p = 0; p < PER; ++p)
#pragma unroll
    for (int i = 0; i < 4; ++i) x.v[p][i] = in_row<G, END>(p, i, lane, d) ? x.v[p][i] - mean : 0.f;
}

// x -> x^ in place.  The variance is taken of the centred row, which keeps its digits where the mean is
// far from zero.
template <int G, RowEnd END, int PER>
__device__ __forceinline__ void normalise(Row<PER>& x, int lane, int d, bool centre, float eps, GroupSum<G>& gs) {
  const float inv_d = 1.0f / static_cast<float>(d);
  if (centre) centre_row<G, END>(x, gs.sum(add_up(x)) * inv_d, lane, d);
  const float r = rsqrtf(gs.sum(dot(x, x)) * inv_d + eps);
#pragma unroll
  for (int p = 0; p < PER; ++p) x.v[p] *= r;
}

// 1 / (1 + e^-z); the reciprocal is the hardware's, within one step of fp32.
__device__ __forceinline__ float sigmoid(float z) { return __builtin_amdgcn_rcpf(1.0f + expf(-z)); }

template <int PER>
__device__ __forceinline__ void sigmoid_row(Row<PER>& g) {
#pragma unroll
  for (int p = 0; p < PER; ++p)
#pragma unroll
    for (int i = 0; i < 4; ++i) g.v[p][i] = sigmoid(g.v[p][i]);
}

// How rows of d elements are dealt to threads: eight elements a thread where the row has them (more in
// flight and in registers lets fewer waves run), four in the shortest rows.  From 4,097 to 8,192 by `fours` fours a
// thread, of 512 (4) or 1,024 (2) threads.
struct RowShape {
  int group, per;
};
inline RowShape row_shape(int d, int fours) {
  if (d <= 256) return {64, 1};
  if (d <= 512) return {64, 2};
  if (d <= 1024) return {256, 1};
  if (d <= 2048) return {256, 2};
  if (d <= 4096) return {512, 2};
  if (d <= 8192) return {2048 / fours, fours};
  return {1024, 4};
}

// Workgroups that hold T rows at once.
inline int row_groups(const RowShape& s, int T) {
  const int rows = s.group == 64 ? 4 : 1;
  return (T + rows - 1) / rows;
}
// Workgroups for T rows, at most `most`, each with as many rows as the others or one fewer.
inline int row_workgroups(const RowShape& s, int T, int most) {
  const int need = row_groups(s, T), turns = (need + most - 1) / most;
  return (need + turns - 1) / turns;
}

// GO(kernel instance, threads) for the row shape, how rows end, and the types of h and y.
#define UMEM_ROW_FULL(KERNEL, HT, YT, G, PER, THR)                                          \
  if (bd.d == 4 * G * PER) UMEM_ROW_GO((KERNEL<HT, YT, G, PER, kFull>), THR);               \
  else if (bd.d % 4 == 0) UMEM_ROW_GO((KERNEL<HT, YT, G, PER, kFours>), THR);               \
  else UMEM_ROW_GO((KERNEL<HT, YT, G, PER, kAny>), THR);
#define UMEM_ROW_SHAPES(KERNEL, HT, YT, FOURS)                              \
  switch (shape.group * 8 + shape.per) {                                    \
    case 64 * 8 + 1: UMEM_ROW_FULL(KERNEL, HT, YT, 64, 1, 256) break;       \
    case 64 * 8 + 2: UMEM_ROW_FULL(KERNEL, HT, YT, 64, 2, 256) break;       \
    case 256 * 8 + 1: UMEM_ROW_FULL(KERNEL, HT, YT, 256, 1, 256) break;     \
    case 256 * 8 + 2: UMEM_ROW_FULL(KERNEL, HT, YT, 256, 2, 256) break;     \
    case 512 * 8 + 2: UMEM_ROW_FULL(KERNEL, HT, YT, 512, 2, 512) break;     \
    case 2048 / FOURS * 8 + FOURS: UMEM_ROW_FULL(KERNEL, HT, YT, 2048 / FOURS, FOURS, 2048 / FOURS) break; \
    default: UMEM_ROW_FULL(KERNEL, HT, YT, 1024, 4, 1024) break;            \
  }
#define UMEM_ROW_LAUNCH(KERNEL, FOURS)                     \
  if (bd.htype == UMEM_F32 && bd.ytype == UMEM_F32) {      \
    UMEM_ROW_SHAPES(KERNEL, float, float, FOURS)                  \
  } else if (bd.htype == UMEM_F32) {                       \
    UMEM_ROW_SHAPES(KERNEL, float, __bf16, FOURS)                 \
  } else if (bd.ytype == UMEM_F32) {                       \
    UMEM_ROW_SHAPES(KERNEL, __bf16, float, FOURS)                 \
  } else {                                                 \
    UMEM_ROW_SHAPES(KERNEL, __bf16, __bf16, FOURS)                \
  }

}  // namespace umem
