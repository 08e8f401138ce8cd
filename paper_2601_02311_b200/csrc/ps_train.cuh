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

// N consecutive elements in the 32-bit words that they were loaded as, by accesses of up to 16 bytes (load, store) or of
// 32 (load32, store32: the address is a multiple of it)
template <class T, int N>
struct Pack {
  static constexpr int WORDS = (N * (int)sizeof(T) + 3) / 4;
  u32 w[WORDS];
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int i = 0; i < WORDS; ++i) w[i] = 0;
  }
  __device__ __forceinline__ void load(const T* p) {
    if (sizeof(T) * N == 2) {
      w[0] = *reinterpret_cast<const unsigned short*>(p);
    } else if (WORDS % 4 == 0) {
#pragma unroll
      for (int i = 0; i < WORDS; i += 4) {
        const uint4 v = reinterpret_cast<const uint4*>(p)[i / 4];
        w[i] = v.x, w[i + 1] = v.y, w[i + 2] = v.z, w[i + 3] = v.w;
      }
    } else if (WORDS % 2 == 0) {
#pragma unroll
      for (int i = 0; i < WORDS; i += 2) {
        const uint2 v = reinterpret_cast<const uint2*>(p)[i / 2];
        w[i] = v.x, w[i + 1] = v.y;
      }
    } else {
#pragma unroll
      for (int i = 0; i < WORDS; ++i) w[i] = reinterpret_cast<const u32*>(p)[i];
    }
  }
  __device__ __forceinline__ void store(T* p) const {
    if (sizeof(T) * N == 2) {
      *reinterpret_cast<unsigned short*>(p) = (unsigned short)w[0];
    } else if (WORDS % 4 == 0) {
#pragma unroll
      for (int i = 0; i < WORDS; i += 4) reinterpret_cast<uint4*>(p)[i / 4] = make_uint4(w[i], w[i + 1], w[i + 2], w[i + 3]);
    } else if (WORDS % 2 == 0) {
#pragma unroll
      for (int i = 0; i < WORDS; i += 2) reinterpret_cast<uint2*>(p)[i / 2] = make_uint2(w[i], w[i + 1]);
    } else {
#pragma unroll
      for (int i = 0; i < WORDS; ++i) reinterpret_cast<u32*>(p)[i] = w[i];
    }
  }
  __device__ __forceinline__ void load32(const T* p) {
    static_assert(WORDS == 8, "32 bytes");
    asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]), "=r"(w[4]), "=r"(w[5]), "=r"(w[6]), "=r"(w[7])
                 : "l"(p));
  }
  __device__ __forceinline__ void store32(T* p) const {
    static_assert(WORDS == 8, "32 bytes");
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
                 ::"l"(p), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]), "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7])
                 : "memory");
  }
  // for results that this kernel does not read again: they are the first to leave the L2
  __device__ __forceinline__ void store32_passing(T* p) const {
    static_assert(WORDS == 8, "32 bytes");
    asm volatile("st.global.L1::no_allocate.L2::evict_first.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
                 ::"l"(p), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]), "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7]) : "memory");
  }
  __device__ __forceinline__ void store_passing(T* p) const {
    if (WORDS % 4 == 0) {
#pragma unroll
      for (int i = 0; i < WORDS; i += 4) __stcs(reinterpret_cast<uint4*>(p) + i / 4, make_uint4(w[i], w[i + 1], w[i + 2], w[i + 3]));
    } else {
      store(p);
    }
  }
  __device__ __forceinline__ void widen(float (&v)[N]) const {
#pragma unroll
    for (int e = 0; e < N; ++e) v[e] = one(w, e, (const T*)nullptr);
  }
  __device__ __forceinline__ void narrow(const float (&v)[N]) {
    if (sizeof(T) == 4) {
#pragma unroll
      for (int e = 0; e < N; ++e) w[e] = __float_as_uint(v[e]);
    } else {
#pragma unroll
      for (int e = 0; e < N; e += 2) w[e / 2] = two(v[e], e + 1 < N ? v[e + 1 < N ? e + 1 : e] : 0.f, (const T*)nullptr);
    }
  }

 private:
  __device__ static __forceinline__ float one(const u32* w, int e, const float*) { return __uint_as_float(w[e]); }
  __device__ static __forceinline__ float one(const u32* w, int e, const __nv_bfloat16*) {
    return __uint_as_float(e & 1 ? w[e / 2] & 0xffff0000u : w[e / 2] << 16);
  }
  __device__ static __forceinline__ float one(const u32* w, int e, const __half*) {
    return __half2float(__ushort_as_half((unsigned short)(e & 1 ? w[e / 2] >> 16 : w[e / 2])));
  }
  __device__ static __forceinline__ u32 two(float, float, const float*) { return 0; }
  __device__ static __forceinline__ u32 two(float lo, float hi, const __nv_bfloat16*) {
    u32 r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
  }
  __device__ static __forceinline__ u32 two(float lo, float hi, const __half*) {
    u32 r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
  }
};

// ---- A chain of kernels of one call.  A kernel that is started by launch_next may begin while the kernel before it in the
// stream still runs: as soon as each block of that one has called let_next_begin (or ended).  What it reads of earlier kernels it reads
// behind wait_for_earlier, which returns once they are done and their results visible (k_queries of ps_attention.cu reads some of it
// earlier, by an order of its own: publish_rows).
__device__ __forceinline__ void let_next_begin() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void wait_for_earlier() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
template <class... Parameters, class... Arguments>
cudaError_t launch_next(void (*kernel)(Parameters...), dim3 grid, u32 threads, u32 smem, cudaStream_t stream, const Arguments&... arguments) {
  cudaLaunchAttribute early;
  early.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  early.val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t config = {};
  config.gridDim = grid;
  config.blockDim = dim3(threads);
  config.dynamicSmemBytes = smem;
  config.stream = stream;
  config.attrs = &early;
  config.numAttrs = 1;
  return cudaLaunchKernelEx(&config, kernel, Parameters(arguments)...);
}

// whether `p` and rows `stride` elements apart begin at multiples of `bytes`
inline bool aligned_rows(const void* p, u64 stride, size_t width, size_t bytes) {
  return reinterpret_cast<uintptr_t>(p) % bytes == 0 && (stride * width) % bytes == 0;
}
// whether packs of n elements may be used at `p` and at rows `stride` elements apart
inline bool packs_at(const void* p, u64 stride, int n, size_t width) {
  const size_t bytes = n * width < 16 ? n * width : 16;
  return aligned_rows(p, stride, width, bytes);
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
