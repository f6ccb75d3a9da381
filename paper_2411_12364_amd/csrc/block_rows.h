// Rows of a residual stream in the registers of a group of threads (block.hip): the loads, stores and
// sums that the norms before and after a block share.  Not part of the public ABI.
#pragma once

#include "umem_internal.h"

namespace umem {

typedef float bf32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bb16x4 __attribute__((ext_vector_type(4)));

// A row's elements are dealt to the G threads of its group in runs of four: element
// (p G + lane) 4 + i is v[p][i] of thread `lane`.  Elements past the row are zeros.
template <int PER>
struct RowRegs {
  bf32x4 v[PER];
};

__device__ __forceinline__ bf32x4 widen(bf32x4 x) { return x; }
__device__ __forceinline__ bf32x4 widen(bb16x4 x) {
  return bf32x4{static_cast<float>(x.x), static_cast<float>(x.y), static_cast<float>(x.z), static_cast<float>(x.w)};
}
template <typename T>
struct Four;
template <>
struct Four<float> {
  using type = bf32x4;
};
template <>
struct Four<__bf16> {
  using type = bb16x4;
};

// VEC: d % 4 == 0 and rows aligned to four elements; else the elements are taken one by one.
template <bool VEC, typename T>
__device__ __forceinline__ bf32x4 load4(const T* row, int e, int d) {
  if constexpr (VEC) {
    if (e >= d) return bf32x4{0.f, 0.f, 0.f, 0.f};
    return widen(*reinterpret_cast<const typename Four<T>::type*>(row + e));
  } else {
    bf32x4 r;
#pragma unroll
    for (int i = 0; i < 4; ++i) r[i] = e + i < d ? static_cast<float>(row[e + i]) : 0.f;
    return r;
  }
}

template <bool VEC, typename T>
__device__ __forceinline__ void store4(T* row, int e, int d, bf32x4 x) {
  const typename Four<T>::type r = {static_cast<T>(x.x), static_cast<T>(x.y), static_cast<T>(x.z), static_cast<T>(x.w)};
  if constexpr (VEC) {
    if (e < d) *reinterpret_cast<typename Four<T>::type*>(row + e) = r;
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (e + i < d) row[e + i] = r[i];
  }
}

template <int G, int PER, bool VEC, typename T>
__device__ __forceinline__ RowRegs<PER> load_row(const T* row, int lane, int d) {
  RowRegs<PER> r;
#pragma unroll
  for (int p = 0; p < PER; ++p) r.v[p] = load4<VEC>(row, (p * G + lane) * 4, d);
  return r;
}

// The sums of up to two values over a group: a wave by shuffles, a workgroup of G threads by its
// waves' sums in LDS, added in wave order by every thread (the same bits in all of them).  `turn`
// picks one of two LDS buffers, so that one barrier a sum is enough.
template <int G>
struct GroupSum {
  static constexpr int kWaves = G / kWave;
  float (*lds)[2][kWaves];            // [2][2][kWaves]
  int turn;

  __device__ __forceinline__ void sum2(float& a, float& b) {
    a = wave_sum(a);
    b = wave_sum(b);
    if constexpr (kWaves > 1) {
      const int wave = threadIdx.x / kWave;
      if ((threadIdx.x & (kWave - 1)) == 0) {
        lds[turn][0][wave] = a;
        lds[turn][1][wave] = b;
      }
      __syncthreads();
      a = b = 0.f;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) {
        a += lds[turn][0][w];
        b += lds[turn][1][w];
      }
      turn ^= 1;
    }
  }
  __device__ __forceinline__ float sum(float a) {
    a = wave_sum(a);
    if constexpr (kWaves > 1) {
      const int wave = threadIdx.x / kWave;
      if ((threadIdx.x & (kWave - 1)) == 0) lds[turn][0][wave] = a;
      __syncthreads();
      a = 0.f;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) a += lds[turn][0][w];
      turn ^= 1;
    }
    return a;
  }
};

// x -> x^ in place (elements past the row stay zero); returns 1 / spread.  The variance is taken of
// the centred row, which keeps its digits where the mean is far from zero.
template <int G, int PER>
__device__ __forceinline__ float normalise(RowRegs<PER>& x, int lane, int d, bool centre, float eps, GroupSum<G>& gs) {
  const float inv_d = 1.0f / static_cast<float>(d);
  if (centre) {
    float s = 0.f;
#pragma unroll
    for (int p = 0; p < PER; ++p) s += (x.v[p].x + x.v[p].y) + (x.v[p].z + x.v[p].w);
    const float mean = gs.sum(s) * inv_d;
#pragma unroll
    for (int p = 0; p < PER; ++p)
#pragma unroll
      for (int i = 0; i < 4; ++i) x.v[p][i] = (p * G + lane) * 4 + i < d ? x.v[p][i] - mean : 0.f;
  }
  float q = 0.f;
#pragma unroll
  for (int p = 0; p < PER; ++p)
#pragma unroll
    for (int i = 0; i < 4; ++i) q = fmaf(x.v[p][i], x.v[p][i], q);
  const float r = 1.0f / sqrtf(gs.sum(q) * inv_d + eps);
#pragma unroll
  for (int p = 0; p < PER; ++p)
#pragma unroll
    for (int i = 0; i < 4; ++i) x.v[p][i] *= r;
  return r;
}

}  // namespace umem
