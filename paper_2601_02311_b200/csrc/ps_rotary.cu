// Rotary positions: pair (a, b) of a head becomes magnitude (a cos t - b sin t, b cos t + a sin t) with t = (position + first) f.
//
// An angle is a whole number of 2^-64 turns: f / 2 pi is rounded to one, and its product with a position, which wraps around,
// is exact however far the position.  The nearest quarter turn is taken off in whole numbers too, so that what becomes a
// float is at most an eighth of a turn and keeps 24 bits of itself.
//
// Bytes bound it: all heads of a token share its angles, so a block computes the sines and cosines of its few tokens once, into
// shared memory, and a thread keeps those of its place in the head in registers while it goes over the heads, 16 bytes at a time, several in flight.
// 2 x 32768 tokens, 64 and 8 heads of 128 in bfloat16, 2.4 GB: 401 us, 6.0 TB/s (0.92 of a copy's rate); with an item's place computed for each, 519 us.
#include <algorithm>
#include "ps_train.cuh"

namespace {
using namespace train;

constexpr int THREADS = 256, TOKENS_MOST = 16;

__device__ __forceinline__ float2 turned(u64 turns, float magnitude) {
  const u64 quarter = (turns + ((u64)1 << 61)) >> 62;
  float s, c;
  sincospif((float)(s64)(turns - (quarter << 62)) * 0x1p-63f, &s, &c);
  const float2 v = quarter & 1 ? make_float2(-s, c) : make_float2(c, s);
  return quarter & 2 ? make_float2(-v.x * magnitude, -v.y * magnitude) : make_float2(v.x * magnitude, v.y * magnitude);
}

// (a, b) turned.  (In roundings of its own, so that every kernel below has the same bits.)
__device__ __forceinline__ void turn(float& a, float& b, float2 circle) {
  const float x = fmaf(a, circle.x, -__fmul_rn(b, circle.y));
  b = fmaf(b, circle.x, __fmul_rn(a, circle.y));
  a = x;
}

// A thread has a place in the head (an item: two packs that turn, one interleaved, or one that is copied) and goes over the heads of a token that its
// place is repeated for, then to the next token: the angles' sines and cosines stay in registers over the heads.
struct Plan {
  u32 tokens, a_block;          // all of them, and a block's
  u32 heads;                    // of q and k
  u32 items, turning;           // of a head, and those of them that turn
  u32 heads_at_once, tokens_at_once;
  Divider by_len;
};

// N elements at a time.  (N = 1: elements or pairs at any alignment.)
template <class T, int N, bool INTERLEAVED>
__global__ void __launch_bounds__(THREADS, 4) k_rotary(const __grid_constant__ RotaryArgs a, const Plan plan) {
  extern __shared__ float2 circle[];                        // [a_block][pairs]: cosine, sine
  const u32 begin = blockIdx.x * plan.a_block, count = min(plan.a_block, plan.tokens - begin);
  for (u32 i = threadIdx.x; i < count * a.pairs; i += THREADS) {
    const u32 t = i / a.pairs, pair = i - t * a.pairs, token = begin + t;
    const u32 b = plan.by_len.of(token), at = token - b * a.len;
    s64 position = at;
    if (a.positions) {
      const u64 where = b * a.position_stride + at;
      position = a.position_bytes == 8 ? ((const s64*)a.positions)[where] : (s64)((const int*)a.positions)[where];
    }
    const u64 turns = ((u64)position + (u64)a.first) * a.turns[pair];
    circle[i] = turned(a.inverse ? 0 - turns : turns, a.magnitude);
  }
  const u32 a_token = plan.items * plan.heads_at_once, slot = threadIdx.x / a_token, place = threadIdx.x - slot * a_token;
  const u32 first = place / plan.items, item = place - first * plan.items;
  const bool turns = item < plan.turning;
  constexpr bool SECOND = !(INTERLEAVED && N > 1);          // an item that turns has two parts
  constexpr int PAIRS = SECOND ? N : N / 2, AT_ONCE = SECOND ? 3 : 6;
  // first element, that of the second part, and first pair
  const u32 column = turns ? (INTERLEAVED && N == 1 ? 2 * item : item * N) : 2 * a.pairs + (item - plan.turning) * N;
  const u32 apart = INTERLEAVED ? 1 : a.pairs, pair = INTERLEAVED ? column / 2 : column;
  __syncthreads();
  if (slot >= plan.tokens_at_once) return;
  for (u32 t = slot; t < count; t += plan.tokens_at_once) {
    const u32 b = plan.by_len.of(begin + t), i = begin + t - b * a.len;
    const T* const q = (const T*)a.q.data + b * a.q.batch_stride + i * a.q.token_stride + column;
    const T* const k = (const T*)a.k.data + b * a.k.batch_stride + i * a.k.token_stride + column;
    T* const q_out = (T*)a.q_out.data + b * a.q_out.batch_stride + i * a.q_out.token_stride + column;
    T* const k_out = (T*)a.k_out.data + b * a.k_out.batch_stride + i * a.k_out.token_stride + column;
    float2 cs[PAIRS];
    if (turns)
#pragma unroll
      for (int e = 0; e < PAIRS; ++e) cs[e] = circle[t * a.pairs + pair + e];
    for (u32 h = first; h < plan.heads; h += AT_ONCE * plan.heads_at_once) {
      Pack<T, N> x[AT_ONCE], y[AT_ONCE];
#pragma unroll
      for (int u = 0; u < AT_ONCE; ++u) {
        const u32 head = h + u * plan.heads_at_once;
        if (head < plan.heads) {
          const T* const from = head < a.heads ? q + head * a.q.head_stride : k + (head - a.heads) * a.k.head_stride;
          x[u].load(from);
          if (SECOND && turns) y[u].load(from + apart);
        }
      }
#pragma unroll
      for (int u = 0; u < AT_ONCE; ++u) {
        const u32 head = h + u * plan.heads_at_once;
        if (head < plan.heads) {
          T* const to = head < a.heads ? q_out + head * a.q_out.head_stride : k_out + (head - a.heads) * a.k_out.head_stride;
          if (turns) {
            float v[N], w[N];
            x[u].widen(v);
            if (SECOND) {
              y[u].widen(w);
#pragma unroll
              for (int e = 0; e < N; ++e) turn(v[e], w[e], cs[SECOND ? e : 0]);
              y[u].narrow(w);
              y[u].store(to + apart);
            } else {
#pragma unroll
              for (int e = 0; e + 1 < N; e += 2) turn(v[e], v[e + 1], cs[e / 2]);
            }
            x[u].narrow(v);
          }
          x[u].store(to);
        }
      }
    }
  }
}

template <class T, int N, bool INTERLEAVED>
cudaError_t rotary(RotaryArgs a, int sm_count, cudaStream_t stream) {
  const auto same = [](const ps_heads& x, const ps_heads& y) {
    return x.data == y.data && x.batch_stride == y.batch_stride && x.token_stride == y.token_stride && x.head_stride == y.head_stride;
  };
  // in its place, what does not turn is left alone
  const bool in_place = same(a.q, a.q_out) && (a.kv_heads == 0 || same(a.k, a.k_out));
  Plan plan;
  plan.heads = a.heads + a.kv_heads;
  plan.turning = (INTERLEAVED && N > 1 ? 2 * a.pairs : a.pairs) / N;
  plan.items = plan.turning + (in_place ? 0 : (a.dim - 2 * a.pairs) / N);
  plan.by_len = Divider(a.len);
  plan.heads_at_once = std::min(plan.heads, THREADS / plan.items);
  plan.tokens_at_once = THREADS / (plan.items * plan.heads_at_once);
  // tokens of a block: a few, but so that all SMs have some blocks
  const u64 tokens = (u64)a.batch * a.len;
  plan.a_block = (u32)std::min<u64>(TOKENS_MOST, std::max<u64>(1, tokens / (8 * (u64)sm_count)));
  // a launch for sequences of up to 2^30 tokens together
  const u32 sequences = std::max(1u, (1u << 30) / a.len);
  for (u32 b = 0; b < a.batch; b += sequences) {
    RotaryArgs p = a;
    p.batch = std::min(sequences, a.batch - b);
    for (ps_heads* h : {&p.q, &p.q_out, &p.k, &p.k_out})
      if (h->data) h->data = (T*)h->data + b * h->batch_stride;
    if (p.positions) p.positions = (const char*)p.positions + b * p.position_stride * p.position_bytes;
    plan.tokens = p.batch * p.len;
    k_rotary<T, N, INTERLEAVED><<<(plan.tokens + plan.a_block - 1) / plan.a_block, THREADS, plan.a_block * a.pairs * sizeof(float2), stream>>>(p, plan);
    const cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return e;
  }
  return cudaSuccess;
}
template <class T>
cudaError_t rotary(const RotaryArgs& a, int sm_count, cudaStream_t stream) {
  constexpr u32 N = 16 / sizeof(T);
  const auto packs = [&](const ps_heads& h) {
    return reinterpret_cast<uintptr_t>(h.data) % 16 == 0 && h.batch_stride % N == 0 && h.token_stride % N == 0 && h.head_stride % N == 0;
  };
  const bool wide = a.dim % N == 0 && (a.interleaved ? 2 * a.pairs : a.pairs) % N == 0 && packs(a.q) && packs(a.q_out) &&
                    (a.kv_heads == 0 || (packs(a.k) && packs(a.k_out)));
  if (wide) return a.interleaved ? rotary<T, N, true>(a, sm_count, stream) : rotary<T, N, false>(a, sm_count, stream);
  return a.interleaved ? rotary<T, 1, true>(a, sm_count, stream) : rotary<T, 1, false>(a, sm_count, stream);
}

}  // namespace

cudaError_t launch_rotary(u32 dtype, const RotaryArgs& a, int sm_count, cudaStream_t stream) {
  if (dtype == PS_F32) return rotary<float>(a, sm_count, stream);
  return dtype == PS_BF16 ? rotary<__nv_bfloat16>(a, sm_count, stream) : rotary<__half>(a, sm_count, stream);
}
