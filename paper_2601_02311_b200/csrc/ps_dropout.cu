// Dropout whose mask is never stored: whether an element is kept is a function of its index in the
// whole tensor, a seed and a stream number, so the backward pass, a recomputation and a shard of
// the tensor on another device all find the mask of the forward pass again.
//
//   y[r, c] = (word(first + r * pitch + c) >= threshold ? x[r, c] * scale : 0) + residual[r, c]
//
// word(g) is word g mod 4 of the counter-based generator Philox4x32-10 (Salmon, Moraes, Dror, Shaw:
// "Parallel Random Numbers: As Easy as 1, 2, 3", 2011) at the counter (g / 4, stream) under the
// key seed; threshold = round(p * 2^32) and scale = 1 / (1 - p).
#include "ps_train.cuh"

namespace {
using namespace train;

struct Words {
  u32 w[4];
};

__device__ __forceinline__ Words philox(u64 counter, u64 stream, u64 seed) {
  u32 a = (u32)counter, b = (u32)(counter >> 32), c = (u32)stream, d = (u32)(stream >> 32);
  u32 k0 = (u32)seed, k1 = (u32)(seed >> 32);
#pragma unroll
  for (int round = 0; round < 10; ++round) {
    const u64 p = (u64)a * 0xD2511F53u, q = (u64)c * 0xCD9E8D57u;
    a = (u32)(q >> 32) ^ b ^ k0;
    b = (u32)q;
    c = (u32)(p >> 32) ^ d ^ k1;
    d = (u32)p;
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
  return {{a, b, c, d}};
}

// one thread, one element
template <class T>
__global__ void k_dropout(DropoutArgs a) {
  const u64 n = a.rows * a.cols;
  for (u64 i = (u64)blockIdx.x * blockDim.x + threadIdx.x; i < n; i += (u64)gridDim.x * blockDim.x) {
    const u64 r = i / a.cols, c = i - r * a.cols, g = a.first + r * a.pitch + c;
    const Words w = philox(g >> 2, a.stream, a.seed);
    float y = (u64)w.w[g & 3] >= a.threshold ? widen(((const T*)a.x)[r * a.x_stride + c]) * a.scale : 0.f;
    if (a.residual) y += widen(((const T*)a.residual)[r * a.residual_stride + c]);
    ((T*)a.y)[r * a.y_stride + c] = narrow<T>(y);
  }
}

}  // namespace

cudaError_t launch_dropout(u32 dtype, const DropoutArgs& a, int sm_count, cudaStream_t stream) {
  const u64 blocks = (a.rows * a.cols + 255) / 256, most = (u64)sm_count * 8;
  const u32 grid = (u32)(blocks < most ? blocks : most);
  if (dtype == PS_F32) k_dropout<float><<<grid, 256, 0, stream>>>(a);
  else if (dtype == PS_BF16) k_dropout<__nv_bfloat16><<<grid, 256, 0, stream>>>(a);
  else k_dropout<__half><<<grid, 256, 0, stream>>>(a);
  return cudaGetLastError();
}
