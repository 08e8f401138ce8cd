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

struct Keep {
  u32 least;        // the smallest word that keeps its element; where threshold is 2^32, none does
  bool none;
  float scale;
  __device__ __forceinline__ explicit Keep(const DropoutArgs& a)
      : least((u32)a.threshold), none(a.threshold >> 32), scale(a.scale) {}
  __device__ __forceinline__ float of(u32 word, float x) const { return word >= least && !none ? x * scale : 0.f; }
};

// A thread takes N consecutive elements (16 bytes, or 8 elements with half a load each) at a time; rows, strides and the
// first element's index are such that packs are aligned in memory and begin with a word 0.
template <class T, int N, bool RESIDUAL>
__global__ void __launch_bounds__(256) k_packs(DropoutArgs a, u32 per_row, Divider by_row, u32 packs) {
  const Keep keep(a);
  for (u32 i = blockIdx.x * 256 + threadIdx.x; i < packs; i += gridDim.x * 256) {
    const u32 r = by_row.of(i);
    const u64 c = (u64)(i - r * per_row) * N;
    Pack<T, N> x, y;
    float v[N], add[N];
    x.load((const T*)a.x + r * a.x_stride + c);
    if (RESIDUAL) y.load((const T*)a.residual + r * a.residual_stride + c);
    const u64 counter = (a.first + r * a.pitch + c) >> 2;
    Words words[N / 4];
#pragma unroll
    for (int q = 0; q < N / 4; ++q) words[q] = philox(counter + q, a.stream, a.seed);
    x.widen(v);
    if (RESIDUAL) y.widen(add);
#pragma unroll
    for (int e = 0; e < N; ++e) {
      v[e] = keep.of(words[e / 4].w[e % 4], v[e]);
      if (RESIDUAL) v[e] += add[e];
    }
    y.narrow(v);
    y.store((T*)a.y + r * a.y_stride + c);
  }
}

// Any alignment: a thread takes the elements of a row that share a counter, element by element.
template <class T, bool RESIDUAL>
__global__ void __launch_bounds__(256) k_groups(DropoutArgs a, u32 per_row, Divider by_row, u32 groups) {
  const Keep keep(a);
  for (u32 i = blockIdx.x * 256 + threadIdx.x; i < groups; i += gridDim.x * 256) {
    const u32 r = by_row.of(i);
    const u64 begin = a.first + r * a.pitch, counter = (begin >> 2) + (i - r * per_row);
    const s64 c = (s64)(counter * 4 - begin);             // of word 0: the first group may begin before the row
    float x[4], y[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (c + e >= 0 && c + e < (s64)a.cols) {
        x[e] = widen(((const T*)a.x)[(s64)(r * a.x_stride) + c + e]);
        if (RESIDUAL) y[e] = widen(((const T*)a.residual)[(s64)(r * a.residual_stride) + c + e]);
      }
    const Words w = philox(counter, a.stream, a.seed);
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (c + e >= 0 && c + e < (s64)a.cols) ((T*)a.y)[(s64)(r * a.y_stride) + c + e] = narrow<T>(keep.of(w.w[e], x[e]) + y[e]);
  }
}

template <class T, bool RESIDUAL>
cudaError_t dropout(DropoutArgs a, int sm_count, cudaStream_t stream) {
  constexpr int N = 16 / sizeof(T);
  const bool together = a.rows == 1 || (a.pitch == a.cols && a.x_stride == a.cols && a.y_stride == a.cols &&
                                        (!RESIDUAL || a.residual_stride == a.cols));
  if (together) {               // rows that follow one another in every sense are one row
    a.cols *= a.rows;
    a.rows = 1;
    a.pitch = a.x_stride = a.y_stride = a.residual_stride = 0;
  }
  const bool packs = a.cols % N == 0 && a.first % 4 == 0 && a.pitch % 4 == 0 && packs_at(a.x, a.x_stride, N, sizeof(T)) &&
                     packs_at(a.y, a.y_stride, N, sizeof(T)) && (!RESIDUAL || packs_at(a.residual, a.residual_stride, N, sizeof(T)));
  // a launch for up to 2^31 items: whole rows, or of a single row a part (2^32 elements, a multiple of N and of 4)
  const u64 part = (u64)1 << 32;
  const u64 cols = a.rows == 1 && a.cols > part ? part : a.cols;
  const u64 per_row = packs ? cols / N : cols / 4 + 2;
  if (per_row > 0x7fffffffu) return cudaErrorInvalidValue;        // (cols above 2^32 in rows of a larger tensor are refused before)
  const u64 rows = 0x7fffffffu / per_row;
  for (u64 r = 0; r < a.rows; r += rows)
    for (u64 c = 0; c < a.cols; c += cols) {
      DropoutArgs p = a;
      p.rows = a.rows - r < rows ? a.rows - r : rows;
      p.cols = a.cols - c < cols ? a.cols - c : cols;
      p.first = a.first + r * a.pitch + c;
      p.x = (const T*)a.x + r * a.x_stride + c;
      if (RESIDUAL) p.residual = (const T*)a.residual + r * a.residual_stride + c;
      p.y = (T*)a.y + r * a.y_stride + c;
      const u32 n = packs ? (u32)(p.cols / N) : (u32)(p.cols / 4 + 2), items = (u32)p.rows * n;
      const u64 blocks = ((u64)items + 255) / 256, most = (u64)sm_count * 8;
      const u32 grid = (u32)(blocks < most ? blocks : most);
      if (packs) k_packs<T, N, RESIDUAL><<<grid, 256, 0, stream>>>(p, n, Divider(n), items);
      else k_groups<T, RESIDUAL><<<grid, 256, 0, stream>>>(p, n, Divider(n), items);
      const cudaError_t e = cudaGetLastError();
      if (e != cudaSuccess) return e;
    }
  return cudaSuccess;
}
template <class T>
cudaError_t dropout(const DropoutArgs& a, int sm_count, cudaStream_t stream) {
  return a.residual ? dropout<T, true>(a, sm_count, stream) : dropout<T, false>(a, sm_count, stream);
}

}  // namespace

cudaError_t launch_dropout(u32 dtype, const DropoutArgs& a, int sm_count, cudaStream_t stream) {
  if (dtype == PS_F32) return dropout<float>(a, sm_count, stream);
  return dtype == PS_BF16 ? dropout<__nv_bfloat16>(a, sm_count, stream) : dropout<__half>(a, sm_count, stream);
}
