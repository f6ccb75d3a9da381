// Low-rank adapters of many requests beside a shared projection:
//   out[t] = base[t] + scale[i] B_i (A_i x[t]),  i = ids[t]
#include <algorithm>

#include "umem_internal.h"

namespace umem {
namespace {

constexpr int THREADS = 256;

struct AdapterArgs {
  const void* x;
  const int32_t* ids;
  const uint16_t *a, *b;
  const float* scale;
  const void* base;
  void* out;
  int T, n, rank, d_in, d_out;
};

typedef uint16_t u16x8 __attribute__((ext_vector_type(8)));

// A workgroup a token: a wave a row of A_i, then a thread an output.
template <typename XT, typename OT>
__global__ __launch_bounds__(THREADS) void adapter_token_kernel(AdapterArgs k) {
  __shared__ float low[kMaxAdapterRank];
  const int t = blockIdx.x, lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
  const int id = k.ids[t];
  const bool on = id >= 0 && id < k.n;
  if (on) {
    const XT* x = static_cast<const XT*>(k.x) + static_cast<size_t>(t) * k.d_in;
    const float scale = k.scale != nullptr ? k.scale[id] : 1.0f;
    for (int r = wave; r < k.rank; r += THREADS / kWave) {
      const uint16_t* a = k.a + (static_cast<size_t>(id) * k.rank + r) * k.d_in;
      float s = 0.f;
      for (int c = lane * 8; c < k.d_in; c += kWave * 8) {
        const u16x8 w = *reinterpret_cast<const u16x8*>(a + c);
#pragma unroll
        for (int i = 0; i < 8; ++i) s = fmaf(bf16_to_f32(w[i]), static_cast<float>(x[c + i]), s);
      }
      s = wave_sum(s);
      if (lane == 0) low[r] = s * scale;
    }
  }
  __syncthreads();
  const OT* base = k.base != nullptr ? static_cast<const OT*>(k.base) + static_cast<size_t>(t) * k.d_out : nullptr;
  OT* out = static_cast<OT*>(k.out) + static_cast<size_t>(t) * k.d_out;
  for (int o = threadIdx.x; o < k.d_out; o += THREADS) {
    float s = 0.f;
    if (on) {
      const uint16_t* b = k.b + (static_cast<size_t>(id) * k.d_out + o) * k.rank;
      for (int r = 0; r < k.rank; r += 8) {
        const u16x8 w = *reinterpret_cast<const u16x8*>(b + r);
#pragma unroll
        for (int i = 0; i < 8; ++i) s = fmaf(bf16_to_f32(w[i]), low[r + i], s);
      }
    }
    out[o] = static_cast<OT>(base != nullptr ? static_cast<float>(base[o]) + s : s);
  }
}

}  // namespace

size_t adapter_workspace_bytes(const umem_adapter_desc& ad, int T) { return 0; }

hipError_t launch_adapter_add(const umem_adapter_desc& ad, int T, const void* x, const int32_t* ids,
                              const uint16_t* a, const uint16_t* b, const float* scale, const void* base,
                              void* out, void* ws, hipStream_t s) {
  clear_stale_error();
  const AdapterArgs k{x, ids, a, b, scale, base, out, T, ad.n, ad.rank, ad.d_in, ad.d_out};
#define UMEM_ADAPTER(XT, OT) \
  hipLaunchKernelGGL((adapter_token_kernel<XT, OT>), dim3(T), dim3(THREADS), 0, s, k)
  if (ad.xtype == UMEM_F32 && ad.otype == UMEM_F32) UMEM_ADAPTER(float, float);
  else if (ad.xtype == UMEM_F32) UMEM_ADAPTER(float, __bf16);
  else if (ad.otype == UMEM_F32) UMEM_ADAPTER(__bf16, float);
  else UMEM_ADAPTER(__bf16, __bf16);
#undef UMEM_ADAPTER
  return hipGetLastError();
}

}  // namespace umem
