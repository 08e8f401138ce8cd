// What the kernels of the training step's operators share: element types and wide accesses.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include "ps_device.cuh"
#include "ps_internal.h"

namespace train {

typedef int64_t s64;

__device__ __forceinline__ float widen(float v) { return v; }
__device__ __forceinline__ float widen(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float widen(__half v) { return __half2float(v); }
template <class T> __device__ __forceinline__ T narrow(float v);     // to nearest even
template <> __device__ __forceinline__ float narrow<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 narrow<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
template <> __device__ __forceinline__ __half narrow<__half>(float v) { return __float2half_rn(v); }

// N consecutive elements, moved in accesses of up to 16 bytes
template <class T, int N>
struct alignas(sizeof(T) * N < 16 ? sizeof(T) * N : 16) Pack {
  T v[N];
};
template <class T, int N>
__device__ __forceinline__ Pack<T, N> load_pack(const T* p) { return *reinterpret_cast<const Pack<T, N>*>(p); }
template <class T, int N>
__device__ __forceinline__ void store_pack(T* p, const Pack<T, N>& v) { *reinterpret_cast<Pack<T, N>*>(p) = v; }

// whether packs of n elements may be used at `p` and at rows `stride` elements apart
inline bool packs_at(const void* p, u64 stride, int n, size_t width) {
  const size_t bytes = n * width < 16 ? n * width : 16;
  return reinterpret_cast<uintptr_t>(p) % bytes == 0 && (stride * width) % bytes == 0;
}

// n / d for n < 2^31 by a product and a shift: with 2^(s - 1) < d <= 2^s and m = ceil(2^(31 + s) / d), n m 2^-(31 + s)
// is off by less than n 2^-31 / d < 1 / d, so its whole part is n / d's; m < 2^32
struct Divider {
  u32 d, m, s;
  Divider() : d(1), m(0), s(0) {}
  explicit Divider(u32 by) : d(by), s(0) {
    while (((u64)1 << s) < by) ++s;
    m = (u32)((((u64)1 << (31 + s)) + by - 1) / by);
  }
  __device__ __forceinline__ u32 of(u32 n) const { return (u32)(((u64)n * m) >> (31 + s)); }
};

}  // namespace train
