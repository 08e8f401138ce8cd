// Sums over the rows of a matrix, column by column, that stand in the same order on every run: blocks leave partial sums in
// 32 bits, parts[n][arrays][cols], and this kernel adds them, first every 32nd part, then the 32 in a tree.
#pragma once
#include "ps_train.cuh"

namespace train {

constexpr int JOIN_COLUMNS = 32, JOIN_SLICES = 32;
template <class O>
__global__ void __launch_bounds__(JOIN_COLUMNS* JOIN_SLICES) k_join_columns(const float* parts, u32 n, u64 cols, O* first, O* second, u32 accumulate) {
  __shared__ float sums[JOIN_SLICES][JOIN_COLUMNS];
  const int lane = threadIdx.x % JOIN_COLUMNS, slice = threadIdx.x / JOIN_COLUMNS;
  const u64 column = (u64)blockIdx.x * JOIN_COLUMNS + lane, pitch = gridDim.y * cols;
  O* const to = blockIdx.y == 0 ? first : second;
  if (to == nullptr) return;                        // (the whole block)
  wait_for_earlier();
  float sum = 0.f;
  if (column < cols) {
    const float* from = parts + blockIdx.y * cols + column;
#pragma unroll 4
    for (u32 i = slice; i < n; i += JOIN_SLICES) sum += from[i * pitch];
  }
  sums[slice][lane] = sum;
  __syncthreads();
#pragma unroll
  for (int half = JOIN_SLICES / 2; half > 0; half /= 2) {
    if (slice < half) sums[slice][lane] += sums[slice + half][lane];
    __syncthreads();
  }
  if (slice == 0 && column < cols) to[column] = narrow<O>(sums[0][lane] + (accumulate ? widen(to[column]) : 0.f));
}

// `first` and `second` (of [cols]; either may be null) from n parts of `arrays` (1 or 2) rows each
template <class O>
cudaError_t join_columns(const float* parts, u32 n, u32 arrays, u64 cols, void* first, void* second, u32 accumulate, cudaStream_t stream) {
  return launch_next(k_join_columns<O>, dim3((u32)((cols + JOIN_COLUMNS - 1) / JOIN_COLUMNS), arrays), JOIN_COLUMNS * JOIN_SLICES, 0, stream, parts, n,
                     cols, (O*)first, (O*)second, accumulate);
}
inline cudaError_t join_columns(u32 dtype, const float* parts, u32 n, u32 arrays, u64 cols, void* first, void* second, u32 accumulate, cudaStream_t stream) {
  if (dtype == PS_F32) return join_columns<float>(parts, n, arrays, cols, first, second, accumulate, stream);
  if (dtype == PS_BF16) return join_columns<__nv_bfloat16>(parts, n, arrays, cols, first, second, accumulate, stream);
  return join_columns<__half>(parts, n, arrays, cols, first, second, accumulate, stream);
}

}  // namespace train
