// Dropout whose mask is never stored: whether an element is kept is a function of its index in the
// whole tensor, a seed and a stream number, so the backward pass, a recomputation and a shard of
// the tensor on another device all find the mask of the forward pass again.
//
//   y[r, c] = (word(first + r * pitch + c) >= threshold ? x[r, c] * scale : 0) + residual[r, c]
//
// word(g) is word g mod 4 of the counter-based generator Philox4x32-10 (Salmon, Moraes, Dror, Shaw:
// "Parallel Random Numbers: As Easy as 1, 2, 3", 2011) at the counter (g / 4, stream) under the
// key seed; threshold = round(p * 2^32) and scale = 1 / (1 - p).
//
// What bounds it: with a residual bytes, 65536 x 8192 in bfloat16, 3.2 GB: 528 us, 6.1 TB/s (0.94 of a copy's rate).  Without one the generator:
// a group of four words is 20 wide products (18 of numbers that depend on the element, 2 of the stream and the seed alone), of which an SM does
// 25 to 32 a cycle, and 20 exclusive-ors, 64 a cycle; 490 us where a copy takes 334.
// Accesses of 32 bytes are fewer instructions: with 16 the two took 567 and 542 us.  12301 x 5003 floats in rows that begin anywhere, 0.49 GB:
// 99 us, 5.0 TB/s; where the tensors' rows do not even lie alike, by accesses of 4 bytes, 118.
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
  __device__ __forceinline__ bool kept(u32 word) const { return word >= least && !none; }
  __device__ __forceinline__ float of(bool kept, float x, float add) const { return fmaf(kept ? x : 0.f, scale, add); }
};

// A thread takes N consecutive elements (16 or 32 bytes) at a time; rows, strides and the first element's index are such that packs
// are aligned in memory and begin with a word 0.
template <class T, int N> constexpr int PACK_BLOCKS = sizeof(T) * N == 32 ? 5 : 8;         // of 256 threads on an SM
template <class T, int N, bool RESIDUAL>
__global__ void __launch_bounds__(256, PACK_BLOCKS<T, N>) k_packs(const DropoutArgs a, const __grid_constant__ Keys keys, u32 per_row, Divider by_row, u32 packs) {
  constexpr bool WIDE = sizeof(T) * N == 32;
  const Keep keep(a);
  for (u32 i = blockIdx.x * 256 + threadIdx.x; i < packs; i += gridDim.x * 256) {
    const u32 r = by_row.of(i);
    const u64 c = (u64)(i - r * per_row) * N, counter = (a.first + r * a.pitch + c) >> 2;
    Pack<T, N> x, y;
    if constexpr (WIDE) {
      x.load32((const T*)a.x + r * a.x_stride + c);
      if (RESIDUAL) y.load32((const T*)a.residual + r * a.residual_stride + c);
    } else {
      x.load((const T*)a.x + r * a.x_stride + c);
      if (RESIDUAL) y.load((const T*)a.residual + r * a.residual_stride + c);
    }
    Words words[N / 4];
#pragma unroll
    for (int q = 0; q < N / 4; ++q) words[q] = philox(counter + q, a.stream, keys);
    float v[N], add[N];
    x.widen(v);
    if (RESIDUAL) y.widen(add);
#pragma unroll
    for (int e = 0; e < N; ++e) v[e] = keep.of(keep.kept(words[e / 4].w[e % 4]), v[e], RESIDUAL ? add[e] : 0.f);
    y.narrow(v);
    if constexpr (WIDE) y.store32((T*)a.y + r * a.y_stride + c);
    else y.store((T*)a.y + r * a.y_stride + c);
  }
}

// Rows that begin anywhere, but in all tensors equally far behind a multiple of 16 bytes: a lane takes such packs, from
// the one in which the row begins on, and an element at the row's ends alone.  A pack's first element is word `phase` of a counter, so its
// last elements' words are of the next lane's counter: the verdicts come from there, a bit each.  A warp takes ROUNDS packs a lane at a time
// but the last lane's last, whose verdicts would be another warp's.  (12301 x 5003 floats: 99 us with 8 packs a lane and two blocks an SM, 103 with 4
// and four, 110 with 8 and three, 130 with 8 and four; k_groups 118.  12301 x 10003 bfloat16: 151 us, k_groups 286.)
constexpr int SHIFTED_BLOCKS = 2;
template <class T> constexpr int SHIFTED_ROUNDS = sizeof(T) == 4 ? 8 : 4;
template <class T> constexpr int SHIFTED_SPAN = (32 * SHIFTED_ROUNDS<T> - 1) * (16 / (int)sizeof(T));
template <class T, bool RESIDUAL>
__global__ void __launch_bounds__(256, SHIFTED_BLOCKS) k_shifted(const DropoutArgs a, const __grid_constant__ Keys keys, u32 per_row, Divider by_row, u32 items) {
  constexpr int N = 16 / sizeof(T), ROUNDS = SHIFTED_ROUNDS<T>, SPAN = SHIFTED_SPAN<T>;
  const Keep keep(a);
  const int lane = threadIdx.x % 32;
  for (u32 item = blockIdx.x * 8 + threadIdx.x / 32; item < items; item += gridDim.x * 8) {
    const u32 r = by_row.of(item), span = item - r * per_row;
    const T* const row = (const T*)a.x + (s64)(r * a.x_stride);
    const s64 cols = (s64)a.cols, column = (s64)span * SPAN - (s64)(reinterpret_cast<uintptr_t>(row) % 16 / sizeof(T));
    const s64 index = (s64)(a.first + r * a.pitch) + column;       // (may be negative, for elements before the row)
    const u32 phase = (u32)index & 3;
    const T* const more = (const T*)a.residual + (s64)(r * a.residual_stride);
    T* const to = (T*)a.y + (s64)(r * a.y_stride);
    Pack<T, N> x[ROUNDS], y[ROUNDS];
    u32 kept[ROUNDS + 1];
    auto first_of = [&](int k) { return column + (32 * k + lane) * N; };
    auto whole = [&](s64 c) { return c >= 0 && c + N <= cols; };
#pragma unroll
    for (int k = 0; k < ROUNDS; ++k) {
      const s64 c = first_of(k);
      x[k].clear();
      y[k].clear();
      if (whole(c)) {
        x[k].load(row + c);
        if (RESIDUAL) y[k].load(more + c);
      }
    }
    kept[ROUNDS] = 0;
#pragma unroll
    for (int k = 0; k < ROUNDS; ++k) {
      kept[k] = 0;
      if (column + 32 * k * N < cols + phase) {
#pragma unroll
        for (int q = 0; q < N / 4; ++q) {
          const Words w = philox((u64)((index >> 2) + (32 * k + lane) * (N / 4) + q), a.stream, keys);
#pragma unroll
          for (int j = 0; j < 4; ++j) kept[k] |= keep.kept(w.w[j]) ? 1u << (4 * q + j) : 0u;
        }
      }
    }
#pragma unroll
    for (int k = 0; k < ROUNDS; ++k) {
      const s64 c = first_of(k);
      const u32 next = __shfl_sync(0xffffffffu, lane == 0 ? kept[k + 1] : kept[k], (lane + 1) % 32);
      const u32 mine = (kept[k] | next << N) >> phase;
      if (k == ROUNDS - 1 && lane == 31) continue;
      if (whole(c)) {
        float v[N], add[N];
        x[k].widen(v);
        if (RESIDUAL) y[k].widen(add);
#pragma unroll
        for (int e = 0; e < N; ++e) v[e] = keep.of(mine >> e & 1, v[e], RESIDUAL ? add[e] : 0.f);
        x[k].narrow(v);
        x[k].store(to + c);
      } else if (c < cols && c + N > 0) {
#pragma unroll 1
        for (int e = 0; e < N; ++e)
          if (c + e >= 0 && c + e < cols)
            to[c + e] = narrow<T>(keep.of(mine >> e & 1, widen(row[c + e]), RESIDUAL ? widen(more[c + e]) : 0.f));
      }
    }
  }
}

// Any alignment: a warp takes SPAN elements of a row at a time, 32 counters for each 128 of them.  A lane draws the four words of a
// counter but moves elements 32 apart, so that a warp's accesses are consecutive; four ballots carry the words' verdicts
// over: bit i of the j-th says whether element 4 i + j is kept.
constexpr int SPAN = 512, RESIDENT_GROUPS = 4;
template <class T, bool RESIDUAL>
__global__ void __launch_bounds__(256, RESIDENT_GROUPS) k_groups(const DropoutArgs a, const __grid_constant__ Keys keys, u32 per_row, Divider by_row, u32 items) {
  const Keep keep(a);
  const int lane = threadIdx.x % 32;
  for (u32 item = blockIdx.x * 8 + threadIdx.x / 32; item < items; item += gridDim.x * 8) {
    const u32 r = by_row.of(item), span = item - r * per_row;
    const u64 begin = a.first + r * a.pitch;
    // elements [low, high) of the SPAN from `column` on are the row's: its first counter may begin before it
    const s64 column = (s64)span * SPAN - (s64)(begin & 3);
    const int low = column < 0 ? (int)-column : 0, high = (int)min((s64)a.cols - column, (s64)SPAN);
    const T* const from = (const T*)a.x + (s64)(r * a.x_stride) + column + lane;
    const T* const more = (const T*)a.residual + (s64)(r * a.residual_stride) + column + lane;
    T* const to = (T*)a.y + (s64)(r * a.y_stride) + column + lane;
    float x[SPAN / 32], add[SPAN / 32];
#pragma unroll
    for (int k = 0; k < SPAN / 32; ++k) {
      x[k] = add[k] = 0.f;
      if (lane + 32 * k >= low && lane + 32 * k < high) {
        x[k] = widen(from[32 * k]);
        if (RESIDUAL) add[k] = widen(more[32 * k]);
      }
    }
#pragma unroll
    for (int q = 0; q < SPAN / 128; ++q) {
      if (128 * q >= high) break;
      const Words w = philox((begin >> 2) + span * (SPAN / 4) + 32 * q + lane, a.stream, keys);
      u32 kept[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) kept[j] = __ballot_sync(0xffffffffu, keep.kept(w.w[j]));
      const u32 mine = (lane & 2 ? (lane & 1 ? kept[3] : kept[2]) : (lane & 1 ? kept[1] : kept[0])) >> (lane / 4);
#pragma unroll
      for (int k = 4 * q; k < 4 * q + 4; ++k)
        if (lane + 32 * k >= low && lane + 32 * k < high) to[32 * k] = narrow<T>(keep.of(mine >> (8 * (k % 4)) & 1, x[k], add[k]));
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
  const bool wide = packs && a.cols % (2 * N) == 0 && aligned_rows(a.x, a.x_stride, sizeof(T), 32) && aligned_rows(a.y, a.y_stride, sizeof(T), 32) &&
                    (!RESIDUAL || aligned_rows(a.residual, a.residual_stride, sizeof(T), 32));
  const auto as_far = [&](const void* p, u64 stride) {         // as far behind a multiple of 16 bytes as x, in every row
    return (reinterpret_cast<uintptr_t>(p) - reinterpret_cast<uintptr_t>(a.x)) % 16 == 0 && (a.rows == 1 || (stride - a.x_stride) * sizeof(T) % 16 == 0);
  };
  const bool shifted = !packs && as_far(a.y, a.y_stride) && (!RESIDUAL || as_far(a.residual, a.residual_stride));
  // a launch for up to 2^31 items: whole rows, or of a single row a part (2^32 elements, a multiple of 2 N and of 4)
  const u64 part = (u64)1 << 32;
  const u64 cols = a.rows == 1 && a.cols > part ? part : a.cols;
  const auto in_row = [&](u64 cols) {
    return packs ? cols / (wide ? 2 * N : N) : shifted ? (cols + N - 1 + SHIFTED_SPAN<T> - 1) / SHIFTED_SPAN<T> : (cols + 3 + SPAN - 1) / SPAN;
  };
  const u64 per_row = in_row(cols);
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
      const u32 n = (u32)in_row(p.cols), items = (u32)p.rows * n;
      const u64 a_block = packs ? 256 : 8, blocks = (items + a_block - 1) / a_block, most = (u64)sm_count * (wide ? PACK_BLOCKS<T, 2 * N> : packs ? PACK_BLOCKS<T, N> : shifted ? SHIFTED_BLOCKS : RESIDENT_GROUPS);
      const u32 grid = (u32)(blocks < most ? blocks : most);
      if (wide) k_packs<T, 2 * N, RESIDUAL><<<grid, 256, 0, stream>>>(p, keys, n, Divider(n), items);
      else if (packs) k_packs<T, N, RESIDUAL><<<grid, 256, 0, stream>>>(p, keys, n, Divider(n), items);
      else if (shifted) k_shifted<T, RESIDUAL><<<grid, 256, 0, stream>>>(p, keys, n, Divider(n), items);
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
