// Layer norm and its gradients.
//
//   y = (x - mean) rstd w + b
//   g = dY w;  xn = (x - mean) rstd;  dX = rstd (g - <g> - xn <g xn>) + residual;  dW = sum_r dY xn;  dB = sum_r dY
//
// with < > the mean over a row.  A row is read once and stays in registers: its mean first, then the sum of squared
// distances from it, so that a large mean costs no digits.  Bytes bound both passes; dW and dB are summed in the
// registers of the threads that own the columns while the rows pass, so that the backward pass reads each matrix once.
//
// Which thread has which columns depends on the width alone: packs of 16 bytes where the width is a multiple of one (read element by
// element where a row does not begin at 16 bytes), elements next to one another where it is not.  So a row's bits do not
// depend on where it lies, nor on the other rows.
#include <algorithm>
#include "ps_columns.cuh"

namespace {
using namespace train;

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int m = 16; m > 0; m /= 2) v += __shfl_xor_sync(0xffffffffu, v, m);
  return v;
}

// Sums over the R threads of a row, the same bits in all of them: within a warp, then over the warps' sums in order.  One barrier a
// call: the next one uses the other half of the slots.
template <int R, int COUNT>
struct RowSum {
  float* slots;         // [2][COUNT][R / 32]
  int turn;
  __device__ __forceinline__ explicit RowSum(float* s) : slots(s), turn(0) {}
  __device__ __forceinline__ void over(float (&v)[COUNT]) {
#pragma unroll
    for (int i = 0; i < COUNT; ++i) v[i] = warp_sum(v[i]);
    if (R == 32) return;
    float* const mine = slots + turn * COUNT * (R / 32);
    turn ^= 1;
    if (threadIdx.x % 32 == 0)
#pragma unroll
      for (int i = 0; i < COUNT; ++i) mine[i * (R / 32) + threadIdx.x / 32] = v[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < COUNT; ++i) v[i] = warp_sum((int)(threadIdx.x % 32) < R / 32 ? mine[i * (R / 32) + threadIdx.x % 32] : 0.f);
  }
};

// E elements of a row in a thread, as R threads share the row
template <class T, int R, int E, bool PACKED>
struct Piece {
  static constexpr int N = PACKED ? 16 / sizeof(T) : 1;       // elements next to one another
  Pack<T, E> p;
  __device__ static __forceinline__ u32 column(int e) { return (e / N * R + threadIdx.x % R) * N + e % N; }
  __device__ static __forceinline__ u32 bits(const float* p) { return __float_as_uint(*p); }
  __device__ static __forceinline__ u32 bits(const __nv_bfloat16* p) { return __bfloat16_as_ushort(*p); }
  __device__ static __forceinline__ u32 bits(const __half* p) { return __half_as_ushort(*p); }
  __device__ __forceinline__ void put(int e, u32 b) {
    if (sizeof(T) == 4) p.w[e] = b;
    else p.w[e / 2] |= b << (16 * (e % 2));
  }
  // `wide`: the row begins at a multiple of 16 bytes.  Columns behind `cols` are zeros.
  __device__ __forceinline__ void load(const T* row, u32 cols, bool wide) {
    p.clear();
    if (PACKED && wide) {
#pragma unroll
      for (int e = 0; e < E; e += N)
        if (column(e) < cols) {
          const uint4 v = *reinterpret_cast<const uint4*>(row + column(e));
          constexpr int W = sizeof(T);      // (words of N elements: 4)
          u32* const to = p.w + e * W / 4;
          to[0] = v.x, to[1] = v.y, to[2] = v.z, to[3] = v.w;
        }
    } else {
#pragma unroll
      for (int e = 0; e < E; ++e)
        if (column(e) < cols) put(e, bits(row + column(e)));
    }
  }
  __device__ __forceinline__ void store(T* row, u32 cols, bool wide) const {
    if (PACKED && wide) {
#pragma unroll
      for (int e = 0; e < E; e += N)
        if (column(e) < cols) {
          const u32* const w = p.w + e * (int)sizeof(T) / 4;
          *reinterpret_cast<uint4*>(row + column(e)) = make_uint4(w[0], w[1], w[2], w[3]);
        }
    } else {
#pragma unroll
      for (int e = 0; e < E; ++e)
        if (column(e) < cols) {
          if (sizeof(T) == 4) reinterpret_cast<u32*>(row)[column(e)] = p.w[e];
          else reinterpret_cast<unsigned short*>(row)[column(e)] = (unsigned short)(p.w[e / 2] >> (16 * (e % 2)));
        }
    }
  }
};

struct Wide {           // which rows begin at multiples of 16 bytes
  bool x, y, d_y, residual, d_x, weight, bias;
};

__host__ __device__ constexpr int threads_of(int r) { return r < 128 ? 128 : r; }

template <class T, int R, int E, bool PACKED>
__global__ void __launch_bounds__(threads_of(R)) k_norm(const NormArgs a, const Wide wide) {
  __shared__ float slots[2 * R / 32];
  RowSum<R, 1> sum(slots);
  constexpr int ROWS = threads_of(R) / R;
  const u32 cols = (u32)a.cols;
  typedef Piece<T, R, E, PACKED> P;
  for (u64 r = (u64)blockIdx.x * ROWS + threadIdx.x / R; r < a.rows; r += (u64)gridDim.x * ROWS) {
    P x, w, b;
    x.load((const T*)a.x.data + r * a.x.stride, cols, wide.x);
    if (a.weight) w.load((const T*)a.weight, cols, wide.weight);
    if (a.bias) b.load((const T*)a.bias, cols, wide.bias);
    float v[E], s[1] = {0.f};
    x.p.widen(v);
#pragma unroll
    for (int e = 0; e < E; ++e) s[0] += v[e];
    sum.over(s);
    const float mean = s[0] / (float)cols;
    s[0] = 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      v[e] = P::column(e) < cols ? v[e] - mean : 0.f;
      s[0] = fmaf(v[e], v[e], s[0]);
    }
    sum.over(s);
    const float rstd = 1.f / sqrtf(s[0] / (float)cols + a.eps);
    float f[E];
    if (a.weight) w.p.widen(f);
#pragma unroll
    for (int e = 0; e < E; ++e) v[e] *= a.weight ? rstd * f[e] : rstd;
    if (a.bias) {
      b.p.widen(f);
#pragma unroll
      for (int e = 0; e < E; ++e) v[e] += f[e];
    }
    x.p.narrow(v);
    x.store((T*)a.y.data + r * a.y.stride, cols, wide.y);
    if (threadIdx.x % R == 0) {
      if (a.mean) a.mean[r] = mean;
      if (a.rstd) a.rstd[r] = rstd;
    }
  }
}

// any width: a block walks the row three times (the second and third time out of the L2)
constexpr int LONG = 1024;
template <class T>
__global__ void __launch_bounds__(LONG) k_norm_long(const NormArgs a) {
  __shared__ float slots[2 * LONG / 32];
  RowSum<LONG, 1> sum(slots);
  for (u64 r = blockIdx.x; r < a.rows; r += gridDim.x) {
    const T* const x = (const T*)a.x.data + r * a.x.stride;
    T* const y = (T*)a.y.data + r * a.y.stride;
    float s[1] = {0.f};
    for (u32 c = threadIdx.x; c < a.cols; c += LONG) s[0] += widen(x[c]);
    sum.over(s);
    const float mean = s[0] / (float)a.cols;
    s[0] = 0.f;
    for (u32 c = threadIdx.x; c < a.cols; c += LONG) {
      const float d = widen(x[c]) - mean;
      s[0] = fmaf(d, d, s[0]);
    }
    sum.over(s);
    const float rstd = 1.f / sqrtf(s[0] / (float)a.cols + a.eps);
    for (u32 c = threadIdx.x; c < a.cols; c += LONG) {
      const float w = a.weight ? widen(((const T*)a.weight)[c]) : 1.f, b = a.bias ? widen(((const T*)a.bias)[c]) : 0.f;
      y[c] = narrow<T>((widen(x[c]) - mean) * (rstd * w) + b);
    }
    if (threadIdx.x == 0) {
      if (a.mean) a.mean[r] = mean;
      if (a.rstd) a.rstd[r] = rstd;
    }
  }
}

// GRADS: the sums over this block's rows for dW and dB go to parts[block][2][cols]
template <class T, int R, int E, bool PACKED, bool GRADS>
__global__ void __launch_bounds__(threads_of(R)) k_norm_grad(const NormArgs a, const Wide wide) {
  constexpr int ROWS = threads_of(R) / R;
  __shared__ float slots[2 * 2 * R / 32];
  __shared__ float joined[ROWS > 1 && GRADS ? 2 * R * E : 1];
  RowSum<R, 2> sum(slots);
  const u32 cols = (u32)a.cols;
  typedef Piece<T, R, E, PACKED> P;
  float of_w[E], of_b[E];
#pragma unroll
  for (int e = 0; e < E; ++e) of_w[e] = of_b[e] = 0.f;
  for (u64 r = (u64)blockIdx.x * ROWS + threadIdx.x / R; r < a.rows; r += (u64)gridDim.x * ROWS) {
    P x, d, w, more;
    x.load((const T*)a.x.data + r * a.x.stride, cols, wide.x);
    d.load((const T*)a.d_y.data + r * a.d_y.stride, cols, wide.d_y);
    if (a.residual.data) more.load((const T*)a.residual.data + r * a.residual.stride, cols, wide.residual);
    if (a.weight) w.load((const T*)a.weight, cols, wide.weight);
    const float mean = a.mean[r], rstd = a.rstd[r];
    float xn[E], g[E], f[E], s[2] = {0.f, 0.f};
    x.p.widen(xn);
    d.p.widen(g);
    if (a.weight) w.p.widen(f);
#pragma unroll
    for (int e = 0; e < E; ++e) {
      xn[e] = (xn[e] - mean) * rstd;
      if (GRADS) {
        of_w[e] = fmaf(g[e], xn[e], of_w[e]);
        of_b[e] += g[e];
      }
      if (a.weight) g[e] *= f[e];
      s[0] += g[e];
      s[1] = fmaf(g[e], xn[e], s[1]);         // (g is 0 behind the last column)
    }
    sum.over(s);
    const float along = s[0] / (float)cols, across = s[1] / (float)cols;
    if (a.residual.data) more.p.widen(f);
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const float v = rstd * (g[e] - fmaf(xn[e], across, along));
      g[e] = a.residual.data ? v + f[e] : v;
    }
    d.p.narrow(g);
    d.store((T*)a.d_x.data + r * a.d_x.stride, cols, wide.d_x);
  }
  if (GRADS) {
    float* const to = a.parts + (u64)blockIdx.x * 2 * cols;
    if (ROWS > 1) {               // the warps' sums, one warp after the other
      for (int turn = 0; turn < ROWS; ++turn) {
        if ((int)(threadIdx.x / R) == turn)
#pragma unroll
          for (int e = 0; e < E; ++e) {
            const u32 at = e * R + threadIdx.x % R;
            of_w[e] += turn ? joined[at] : 0.f;
            of_b[e] += turn ? joined[R * E + at] : 0.f;
            joined[at] = of_w[e];
            joined[R * E + at] = of_b[e];
          }
        __syncthreads();
      }
      if (threadIdx.x / R != ROWS - 1) return;
    }
#pragma unroll
    for (int e = 0; e < E; ++e)
      if (P::column(e) < cols) {
        to[P::column(e)] = of_w[e];
        to[cols + P::column(e)] = of_b[e];
      }
  }
}

// any width: dX by a block a row, in two walks
template <class T>
__global__ void __launch_bounds__(LONG) k_norm_grad_long(const NormArgs a) {
  __shared__ float slots[2 * 2 * LONG / 32];
  RowSum<LONG, 2> sum(slots);
  for (u64 r = blockIdx.x; r < a.rows; r += gridDim.x) {
    const T* const x = (const T*)a.x.data + r * a.x.stride;
    const T* const d_y = (const T*)a.d_y.data + r * a.d_y.stride;
    const T* const more = a.residual.data ? (const T*)a.residual.data + r * a.residual.stride : nullptr;
    T* const d_x = (T*)a.d_x.data + r * a.d_x.stride;
    const float mean = a.mean[r], rstd = a.rstd[r];
    float s[2] = {0.f, 0.f};
    for (u32 c = threadIdx.x; c < a.cols; c += LONG) {
      const float g = widen(d_y[c]) * (a.weight ? widen(((const T*)a.weight)[c]) : 1.f);
      s[0] += g;
      s[1] = fmaf(g, (widen(x[c]) - mean) * rstd, s[1]);
    }
    sum.over(s);
    const float along = s[0] / (float)a.cols, across = s[1] / (float)a.cols;
    for (u32 c = threadIdx.x; c < a.cols; c += LONG) {
      const float g = widen(d_y[c]) * (a.weight ? widen(((const T*)a.weight)[c]) : 1.f);
      const float v = rstd * (g - fmaf((widen(x[c]) - mean) * rstd, across, along));
      d_x[c] = narrow<T>(more ? v + widen(more[c]) : v);
    }
  }
}
// and dW, dB: a block has 256 columns, a thread each, and a chunk of the rows
template <class T>
__global__ void __launch_bounds__(256) k_norm_columns(const NormArgs a, u64 rows_each) {
  const u64 c = (u64)blockIdx.x * 256 + threadIdx.x;
  if (c >= a.cols) return;
  const u64 begin = blockIdx.y * rows_each, end = begin + rows_each < a.rows ? begin + rows_each : a.rows;
  float of_w = 0.f, of_b = 0.f;
#pragma unroll 4
  for (u64 r = begin; r < end; ++r) {
    const float d = widen(((const T*)a.d_y.data)[r * a.d_y.stride + c]);
    of_w = fmaf(d, (widen(((const T*)a.x.data)[r * a.x.stride + c]) - a.mean[r]) * a.rstd[r], of_w);
    of_b += d;
  }
  float* const to = a.parts + (u64)blockIdx.y * 2 * a.cols + c;
  to[0] = of_w;
  to[a.cols] = of_b;
}

// blocks that the rows are spread over, at most
u32 blocks_for(u64 rows, int rows_a_block, int resident, int sm_count) {
  const u64 need = (rows + rows_a_block - 1) / rows_a_block, most = (u64)sm_count * resident;
  return (u32)(need < most ? need : most);
}

// Elements of a thread and threads of a row, by the width: as few threads as hold the row in E registers each.  The
// backward pass has two sums a column beside the row's two matrices, hence fewer columns a thread.
constexpr int E_FORWARD = 32;
template <class T, int R, bool PACKED>
cudaError_t forward(const NormArgs& a, const Wide& wide, int sm_count, cudaStream_t stream) {
  const int threads = threads_of(R), resident = 2048 / threads;
  k_norm<T, R, E_FORWARD, PACKED><<<blocks_for(a.rows, threads / R, resident, sm_count), threads, 0, stream>>>(a, wide);
  return cudaGetLastError();
}
template <class T, bool PACKED>
cudaError_t forward(const NormArgs& a, const Wide& wide, int sm_count, cudaStream_t stream) {
  if (a.cols <= 32 * E_FORWARD) return forward<T, 32, PACKED>(a, wide, sm_count, stream);
  if (a.cols <= 128 * E_FORWARD) return forward<T, 128, PACKED>(a, wide, sm_count, stream);
  if (a.cols <= 256 * E_FORWARD) return forward<T, 256, PACKED>(a, wide, sm_count, stream);
  if (a.cols <= 512 * E_FORWARD) return forward<T, 512, PACKED>(a, wide, sm_count, stream);
  if (a.cols <= 1024 * E_FORWARD) return forward<T, 1024, PACKED>(a, wide, sm_count, stream);
  k_norm_long<T><<<blocks_for(a.rows, 1, 2, sm_count), LONG, 0, stream>>>(a);
  return cudaGetLastError();
}
Wide wide_of(const NormArgs& a, size_t width) {
  const auto at = [&](const ps_matrix& m) { return aligned_rows(m.data, m.stride, width, 16); };
  return {at(a.x), at(a.y), at(a.d_y), at(a.residual), at(a.d_x), aligned_rows(a.weight, 0, width, 16), aligned_rows(a.bias, 0, width, 16)};
}
template <class T>
cudaError_t forward(const NormArgs& a, int sm_count, cudaStream_t stream) {
  const Wide wide = wide_of(a, sizeof(T));
  return a.cols % (16 / sizeof(T)) == 0 ? forward<T, true>(a, wide, sm_count, stream) : forward<T, false>(a, wide, sm_count, stream);
}

// the backward pass's shape: threads of a row (0: the long kernels) and blocks, which are the parts of the sums
struct Shape {
  int threads, elements;
  u32 blocks;
};
// (a number of blocks for 148 SMs, whatever the device has: the sums' order depends on the sizes alone)
constexpr int SMS = 148;
Shape backward_shape(u32 width, u64 rows, u64 cols) {
  Shape s = {0, 16, 0};
  if (width == 2 && cols <= 1024) s.threads = 32, s.elements = 32;
  else if (width == 4 && cols <= 512) s.threads = 32;
  else if (cols <= 2048) s.threads = 128;
  else if (cols <= 4096) s.threads = 256;
  else if (cols <= 8192) s.threads = 512;
  else if (width == 2 && cols <= 16384) s.threads = 512, s.elements = 32;
  if (s.threads == 0) s.blocks = (u32)std::max<u64>(1, std::min<u64>((rows + 63) / 64, 64));          // (chunks of rows)
  else {
    const int block = threads_of(s.threads);
    s.blocks = std::max(1u, blocks_for(rows, block / s.threads, s.elements == 32 && s.threads == 512 ? 1 : 512 / block, SMS));
  }
  return s;
}
template <class T, int R, int E, bool PACKED>
cudaError_t backward(const NormArgs& a, const Wide& wide, const Shape& s, cudaStream_t stream) {
  if (a.parts) k_norm_grad<T, R, E, PACKED, true><<<s.blocks, threads_of(R), 0, stream>>>(a, wide);
  else k_norm_grad<T, R, E, PACKED, false><<<s.blocks, threads_of(R), 0, stream>>>(a, wide);
  return cudaGetLastError();
}
template <class T, bool PACKED>
cudaError_t backward(const NormArgs& a, const Shape& s, int sm_count, cudaStream_t stream) {
  const Wide wide = wide_of(a, sizeof(T));
  constexpr bool HALF = sizeof(T) == 2;
  if (s.threads == 32) return backward<T, 32, HALF ? 32 : 16, PACKED>(a, wide, s, stream);
  if (s.threads == 128) return backward<T, 128, 16, PACKED>(a, wide, s, stream);
  if (s.threads == 256) return backward<T, 256, 16, PACKED>(a, wide, s, stream);
  if (s.threads == 512 && s.elements == 16) return backward<T, 512, 16, PACKED>(a, wide, s, stream);
  if constexpr (HALF)
    if (s.threads == 512) return backward<T, 512, 32, PACKED>(a, wide, s, stream);
  if (a.parts) {                 // before d_x, which may stand in the place of d_y or x
    k_norm_columns<T><<<dim3((u32)((a.cols + 255) / 256), s.blocks), 256, 0, stream>>>(a, (a.rows + s.blocks - 1) / s.blocks);
    const cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return e;
  }
  if (a.rows == 0) return cudaSuccess;
  k_norm_grad_long<T><<<blocks_for(a.rows, 1, 2, sm_count), LONG, 0, stream>>>(a);
  return cudaGetLastError();
}
template <class T>
cudaError_t backward(const NormArgs& a, int sm_count, cudaStream_t stream) {
  const Shape s = backward_shape(sizeof(T), a.rows, a.cols);
  if (a.rows == 0 && !a.parts) return cudaSuccess;
  const cudaError_t e = a.cols % (16 / sizeof(T)) == 0 ? backward<T, true>(a, s, sm_count, stream) : backward<T, false>(a, s, sm_count, stream);
  if (e != cudaSuccess || !a.parts) return e;
  return join_columns(a.grad_dtype, a.parts, s.blocks, 2, a.cols, a.d_weight, a.d_bias, a.accumulate, stream);
}

}  // namespace

cudaError_t launch_norm_forward(u32 dtype, const NormArgs& a, int sm_count, cudaStream_t stream) {
  if (dtype == PS_F32) return forward<float>(a, sm_count, stream);
  return dtype == PS_BF16 ? forward<__nv_bfloat16>(a, sm_count, stream) : forward<__half>(a, sm_count, stream);
}

size_t norm_backward_bytes(u32 dtype, const NormArgs& a) {
  return (size_t)backward_shape(dtype == PS_F32 ? 4 : 2, a.rows, a.cols).blocks * 2 * a.cols * sizeof(float);
}

cudaError_t launch_norm_backward(u32 dtype, const NormArgs& a, int sm_count, cudaStream_t stream) {
  if (dtype == PS_F32) return backward<float>(a, sm_count, stream);
  return dtype == PS_BF16 ? backward<__nv_bfloat16>(a, sm_count, stream) : backward<__half>(a, sm_count, stream);
}
