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

// the keys of the generator's rounds, which depend on the seed alone
struct Keys {
  u32 k[10][2];
  explicit Keys(u64 seed) {
    for (u32 r = 0; r < 10; ++r) {
      k[r][0] = (u32)seed + r * 0x9E3779B9u;
      k[r][1] = (u32)(seed >> 32) + r * 0xBB67AE85u;
    }
  }
};

__device__ __forceinline__ Words philox(u64 counter, u64 stream, const Keys& keys) {
  u32 a = (u32)counter, b = (u32)(counter >> 32), c = (u32)stream, d = (u32)(stream >> 32);
#pragma unroll
  for (int r = 0; r < 10; ++r) {
    const u64 p = (u64)a * 0xD2511F53u, q = (u64)c * 0xCD9E8D57u;
    a = (u32)(q >> 32) ^ b ^ keys.k[r][0];
    b = (u32)q;
    c = (u32)(p >> 32) ^ d ^ keys.k[r][1];
    d = (u32)p;
  }
  return {{a, b, c, d}};
}

struct Keep {
  u32 least;        // the smallest word that keeps its element; where threshold is 2^32, none does
  bool none;
  float scale;
  __device__ __forceinline__ explicit Keep(const DropoutArgs& a)
      : least((u32)a.threshold), none(a.threshold >> 32), scale(a.scale) {}
  __device__ __forceinline__ float of(u32 word, float x, float add) const {
    return fmaf(word >= least && !none ? x : 0.f, scale, add);
  }
};

#ifndef DU
#define DU 1
#endif
#ifndef DB
#define DB 8
#endif
constexpr int UNROLL = DU, RESIDENT = DB;
// A thread takes UNROLL packs of N consecutive elements (16 bytes) at a time, a grid apart; rows, strides and the
// first element's index are such that packs are aligned in memory and begin with a word 0.
template <class T, int N, bool RESIDUAL>
__global__ void __launch_bounds__(256, RESIDENT) k_packs(const DropoutArgs a, const __grid_constant__ Keys keys, u32 per_row, Divider by_row, u32 packs) {
  const Keep keep(a);
  const u32 step = gridDim.x * 256;
  for (u32 i = blockIdx.x * 256 + threadIdx.x; i < packs; i += step * UNROLL) {
    Pack<T, N> x[UNROLL], y[UNROLL];
    u32 row[UNROLL];
    u64 column[UNROLL];
#pragma unroll
    for (int u = 0; u < UNROLL; ++u) {
      const u32 at = i + u * step;
      row[u] = by_row.of(at);
      column[u] = (u64)(at - row[u] * per_row) * N;
      if (at < packs) {
        x[u].load((const T*)a.x + row[u] * a.x_stride + column[u]);
        if (RESIDUAL) y[u].load((const T*)a.residual + row[u] * a.residual_stride + column[u]);
      }
    }
#pragma unroll
    for (int u = 0; u < UNROLL; ++u) {
      const u64 counter = (a.first + row[u] * a.pitch + column[u]) >> 2;
      Words words[N / 4];
      float v[N], add[N];
#pragma unroll
      for (int q = 0; q < N / 4; ++q) words[q] = philox(counter + q, a.stream, keys);
      if (i + u * step < packs) {
        x[u].widen(v);
        if (RESIDUAL) y[u].widen(add);
#pragma unroll
        for (int e = 0; e < N; ++e) v[e] = keep.of(words[e / 4].w[e % 4], v[e], RESIDUAL ? add[e] : 0.f);
        y[u].narrow(v);
        y[u].store((T*)a.y + row[u] * a.y_stride + column[u]);
      }
    }
  }
}

// Any alignment: a thread takes the elements of a row that share a counter, element by element.
template <class T, bool RESIDUAL>
__global__ void __launch_bounds__(256, RESIDENT) k_groups(const DropoutArgs a, const __grid_constant__ Keys keys, u32 per_row, Divider by_row, u32 groups) {
  const Keep keep(a);
  const u32 step = gridDim.x * 256;
  for (u32 i = blockIdx.x * 256 + threadIdx.x; i < groups; i += step * UNROLL) {
    float x[UNROLL][4], y[UNROLL][4];
    u32 row[UNROLL];
    u64 counter[UNROLL];
    s64 column[UNROLL];                                         // of word 0: a row's first group may begin before it
#pragma unroll
    for (int u = 0; u < UNROLL; ++u) {
      const u32 at = i + u * step, r = by_row.of(at);
      const u64 begin = a.first + r * a.pitch;
      row[u] = r;
      counter[u] = (begin >> 2) + (at - r * per_row);
      column[u] = at < groups ? (s64)(counter[u] * 4 - begin) : (s64)a.cols;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const s64 c = column[u] + e;
        x[u][e] = y[u][e] = 0.f;
        if (c >= 0 && c < (s64)a.cols) {
          x[u][e] = widen(((const T*)a.x)[(s64)(r * a.x_stride) + c]);
          if (RESIDUAL) y[u][e] = widen(((const T*)a.residual)[(s64)(r * a.residual_stride) + c]);
        }
      }
    }
#pragma unroll
    for (int u = 0; u < UNROLL; ++u) {
      const Words w = philox(counter[u], a.stream, keys);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const s64 c = column[u] + e;
        if (c >= 0 && c < (s64)a.cols) ((T*)a.y)[(s64)(row[u] * a.y_stride) + c] = narrow<T>(keep.of(w.w[e], x[u][e], y[u][e]));
      }
    }
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
  const Keys keys(a.seed);
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
      const u64 blocks = ((u64)items + 255) / 256, most = (u64)sm_count * RESIDENT;
      const u32 grid = (u32)(blocks < most ? blocks : most);
      if (packs) k_packs<T, N, RESIDUAL><<<grid, 256, 0, stream>>>(p, keys, n, Divider(n), items);
      else k_groups<T, RESIDUAL><<<grid, 256, 0, stream>>>(p, keys, n, Divider(n), items);
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
