// Attention and its backward pass.
//
//   S = scale * Q K^T over the keys a query sees;  lse_i = log sum_j exp(S_ij);  O = exp(S - lse) V
//   delta_i = sum_d dO_id O_id;  P = exp(S - lse);  dS = P o (dO V^T - delta)
//   dQ = scale * dS K;  dK = scale * dS^T Q;  dV = P^T dO       (dK, dV over the query heads of a key head)
//
// Query i of a sequence of n queries and m keys sees key j < m, under the causal mask those with j <= i + m - n.
// A query that sees nothing has O = 0 and lse = -infinity, and no gradient.  Queries behind n and keys behind m are
// padding: nothing of theirs is used, and zeros are written for them.
#include "ps_train.cuh"

namespace {
using namespace train;

constexpr float MINUS_INF = -INFINITY;

template <class T>
__device__ __forceinline__ const T* token_of(const ps_heads& h, u64 b, u64 t, u64 head) {
  return (const T*)h.data + b * h.batch_stride + t * h.token_stride + head * h.head_stride;
}
__device__ __forceinline__ int length_of(const int* lens, int b, int most) { return lens ? max(0, min(lens[b], most)) : most; }
__device__ __forceinline__ float warp_sum(float v) {
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// a token's elements of a head, 4 to a lane (dim <= 128)
struct Row {
  float v[4];
};
template <class T>
__device__ __forceinline__ Row load_row(const T* p, int dim) {
  Row r;
  for (int e = 0; e < 4; ++e) {
    const int c = threadIdx.x % 32 + 32 * e;
    r.v[e] = c < dim ? widen(p[c]) : 0.f;
  }
  return r;
}
template <class T>
__device__ __forceinline__ void store_row(const T* at, const Row& r, int dim, float by) {
  T* p = const_cast<T*>(at);
  for (int e = 0; e < 4; ++e) {
    const int c = threadIdx.x % 32 + 32 * e;
    if (c < dim) p[c] = narrow<T>(r.v[e] * by);
  }
}
__device__ __forceinline__ float dot(const Row& a, const Row& b) {
  float s = 0.f;
  for (int e = 0; e < 4; ++e) s += a.v[e] * b.v[e];
  return warp_sum(s);
}
__device__ __forceinline__ void add(Row& a, const Row& b, float by) {
  for (int e = 0; e < 4; ++e) a.v[e] += b.v[e] * by;
}

// one warp, one query
template <class T>
__global__ void k_attend(AttentionArgs a) {
  const u64 w = ((u64)blockIdx.x * blockDim.x + threadIdx.x) / 32;
  if (w >= (u64)a.batch * a.heads * a.q_len) return;
  const int i = (int)(w % a.q_len), h = (int)(w / a.q_len % a.heads), b = (int)(w / a.q_len / a.heads), kh = h / (a.heads / a.kv_heads);
  const int n = length_of(a.q_lens, b, a.q_len), m = length_of(a.k_lens, b, a.k_len);
  const int end = i >= n ? 0 : a.causal ? min(m, i + m - n + 1) : m;
  const Row q = load_row(token_of<T>(a.q, b, i, h), a.dim);
  Row sum = {};
  float most = MINUS_INF, total = 0.f;
  for (int j = 0; j < end; ++j) {
    const float s = dot(q, load_row(token_of<T>(a.k, b, j, kh), a.dim)) * a.scale;
    const float next = fmaxf(most, s), by = most == MINUS_INF ? 0.f : __expf(most - next);
    const float p = __expf(s - next);
    for (int e = 0; e < 4; ++e) sum.v[e] *= by;
    total = total * by + p;
    most = next;
    add(sum, load_row(token_of<T>(a.v, b, j, kh), a.dim), p);
  }
  store_row(token_of<T>(a.out, b, i, h), sum, a.dim, total > 0.f ? 1.f / total : 0.f);
  if (threadIdx.x % 32 == 0) a.lse[w] = total > 0.f ? most + __logf(total) : MINUS_INF;
}

// one warp, one query: delta and dQ
template <class T>
__global__ void k_query_gradient(AttentionArgs a) {
  const u64 w = ((u64)blockIdx.x * blockDim.x + threadIdx.x) / 32;
  if (w >= (u64)a.batch * a.heads * a.q_len) return;
  const int i = (int)(w % a.q_len), h = (int)(w / a.q_len % a.heads), b = (int)(w / a.q_len / a.heads), kh = h / (a.heads / a.kv_heads);
  const int n = length_of(a.q_lens, b, a.q_len), m = length_of(a.k_lens, b, a.k_len);
  const int end = i >= n ? 0 : a.causal ? min(m, i + m - n + 1) : m;
  const Row q = load_row(token_of<T>(a.q, b, i, h), a.dim), d_out = load_row(token_of<T>(a.d_out, b, i, h), a.dim);
  const float delta = dot(d_out, load_row(token_of<T>(a.out, b, i, h), a.dim)), lse = a.lse[w];
  if (threadIdx.x % 32 == 0) a.delta[w] = delta;
  Row sum = {};
  for (int j = 0; j < end; ++j) {
    const Row k = load_row(token_of<T>(a.k, b, j, kh), a.dim);
    const float p = __expf(dot(q, k) * a.scale - lse);
    add(sum, k, p * (dot(d_out, load_row(token_of<T>(a.v, b, j, kh), a.dim)) - delta));
  }
  store_row(token_of<T>(a.d_q, b, i, h), sum, a.dim, a.scale);
}

// one warp, one key: dK and dV
template <class T>
__global__ void k_key_gradient(AttentionArgs a) {
  const u64 w = ((u64)blockIdx.x * blockDim.x + threadIdx.x) / 32;
  if (w >= (u64)a.batch * a.kv_heads * a.k_len) return;
  const int j = (int)(w % a.k_len), kh = (int)(w / a.k_len % a.kv_heads), b = (int)(w / a.k_len / a.kv_heads), group = a.heads / a.kv_heads;
  const int n = length_of(a.q_lens, b, a.q_len), m = length_of(a.k_lens, b, a.k_len);
  const int begin = j >= m ? n : a.causal ? max(0, j - m + n) : 0;
  const Row k = load_row(token_of<T>(a.k, b, j, kh), a.dim), v = load_row(token_of<T>(a.v, b, j, kh), a.dim);
  Row sum_k = {}, sum_v = {};
  for (int h = kh * group; h < (kh + 1) * group; ++h)
    for (int i = begin; i < n; ++i) {
      const u64 at = ((u64)b * a.heads + h) * a.q_len + i;
      const Row q = load_row(token_of<T>(a.q, b, i, h), a.dim), d_out = load_row(token_of<T>(a.d_out, b, i, h), a.dim);
      const float p = __expf(dot(q, k) * a.scale - a.lse[at]);
      add(sum_v, d_out, p);
      add(sum_k, q, p * (dot(d_out, v) - a.delta[at]));
    }
  store_row(token_of<T>(a.d_k, b, j, kh), sum_k, a.dim, a.scale);
  store_row(token_of<T>(a.d_v, b, j, kh), sum_v, a.dim, 1.f);
}

}  // namespace

cudaError_t launch_attention_forward(u32 dtype, const AttentionArgs& a, int, cudaStream_t stream) {
  const u64 rows = (u64)a.batch * a.heads * a.q_len;
  const u32 grid = (u32)((rows + 7) / 8);
  if (rows == 0) return cudaSuccess;
  if (dtype == PS_BF16) k_attend<__nv_bfloat16><<<grid, 256, 0, stream>>>(a);
  else k_attend<__half><<<grid, 256, 0, stream>>>(a);
  return cudaGetLastError();
}

size_t attention_backward_bytes(const AttentionArgs& a) { return (size_t)a.batch * a.heads * a.q_len * sizeof(float); }

cudaError_t launch_attention_backward(u32 dtype, const AttentionArgs& a, int, cudaStream_t stream) {
  const u64 rows = (u64)a.batch * a.heads * a.q_len, keys = (u64)a.batch * a.kv_heads * a.k_len;
  const u32 grid = (u32)((rows + 7) / 8), grid_k = (u32)((keys + 7) / 8);
  if (dtype == PS_BF16) {
    if (rows) k_query_gradient<__nv_bfloat16><<<grid, 256, 0, stream>>>(a);
    if (keys) k_key_gradient<__nv_bfloat16><<<grid_k, 256, 0, stream>>>(a);
  } else {
    if (rows) k_query_gradient<__half><<<grid, 256, 0, stream>>>(a);
    if (keys) k_key_gradient<__half><<<grid_k, 256, 0, stream>>>(a);
  }
  return cudaGetLastError();
}
