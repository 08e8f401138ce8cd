// The embedding lookup and its gradient.
//
//   out[t]     = scale * table[token[t] - first_row]           (zeros where that row is not held)
//   d_table[v] = scale * sum over t with token[t] - first_row = v, t ascending, of d_out[t]
//
// Sums are held in 32 bits and rounded once.  Which token adds to which row in which order follows from the tokens
// alone, so the gradient has the same bits on every run.
#include "ps_train.cuh"

namespace {
using namespace train;

// the row of the table that token t looks up, or rows where none that is held
__device__ __forceinline__ u32 row_of(const EmbedArgs& a, u64 t) {
  const s64 id = a.token_bytes == 8 ? ((const s64*)a.tokens)[t] : (s64)((const int*)a.tokens)[t];
  const u64 row = (u64)id - a.first_row;
  return id >= 0 && (u64)id >= a.first_row && row < a.rows ? (u32)row : (u32)a.rows;
}

template <class T>
__global__ void k_lookup(EmbedArgs a) {
  for (u64 t = blockIdx.x; t < a.n_tokens; t += gridDim.x) {
    const u32 row = row_of(a, t);
    for (u64 c = threadIdx.x; c < a.dim; c += blockDim.x)
      ((T*)a.out)[t * a.out_stride + c] =
          row < a.rows ? narrow<T>(widen(((const T*)a.table)[row * a.table_stride + c]) * a.scale) : narrow<T>(0.f);
  }
}

// one block, one row of the table
template <class T, class G>
__global__ void k_gradient(EmbedArgs a) {
  for (u64 v = blockIdx.x; v < a.rows; v += gridDim.x)
    for (u64 c = threadIdx.x; c < a.dim; c += blockDim.x) {
      float sum = 0.f;
      for (u64 t = 0; t < a.n_tokens; ++t)
        if (row_of(a, t) == v) sum += widen(((const T*)a.out)[t * a.out_stride + c]);
      G* at = (G*)a.table + v * a.table_stride + c;
      *at = narrow<G>(sum * a.scale + (a.accumulate ? widen(*at) : 0.f));
    }
}

template <class T>
void gradient(u32 grad_dtype, const EmbedArgs& a, u32 grid, cudaStream_t stream) {
  if (grad_dtype == PS_F32) k_gradient<T, float><<<grid, 256, 0, stream>>>(a);
  else if (grad_dtype == PS_BF16) k_gradient<T, __nv_bfloat16><<<grid, 256, 0, stream>>>(a);
  else k_gradient<T, __half><<<grid, 256, 0, stream>>>(a);
}

}  // namespace

cudaError_t launch_embed_forward(u32 dtype, const EmbedArgs& a, int sm_count, cudaStream_t stream) {
  const u64 most = (u64)sm_count * 8;
  const u32 grid = (u32)(a.n_tokens < most ? a.n_tokens : most);
  if (dtype == PS_F32) k_lookup<float><<<grid, 256, 0, stream>>>(a);
  else if (dtype == PS_BF16) k_lookup<__nv_bfloat16><<<grid, 256, 0, stream>>>(a);
  else k_lookup<__half><<<grid, 256, 0, stream>>>(a);
  return cudaGetLastError();
}

size_t embed_backward_bytes(const EmbedArgs&) { return 0; }

cudaError_t launch_embed_backward(u32 dtype, u32 grad_dtype, const EmbedArgs& a, int sm_count, cudaStream_t stream) {
  const u64 most = (u64)sm_count * 8;
  const u32 grid = (u32)(a.rows < most ? a.rows : most);
  if (dtype == PS_F32) gradient<float>(grad_dtype, a, grid, stream);
  else if (dtype == PS_BF16) gradient<__nv_bfloat16>(grad_dtype, a, grid, stream);
  else gradient<__half>(grad_dtype, a, grid, stream);
  return cudaGetLastError();
}
