// Rotary positions: pair (a, b) of a head becomes magnitude (a cos t - b sin t, b cos t + a sin t) with t = (position + first) f.
//
// An angle is a whole number of 2^-64 turns: f / 2 pi is rounded to one, and its product with a position, which wraps around,
// is exact however far the position.  The nearest quarter turn is taken off in whole numbers too, so that what becomes a
// float is at most an eighth of a turn and keeps 24 bits of itself.
//
// Bytes bound it: all heads of a token share its angles, so a block computes the sines and cosines of its few tokens once, into
// shared memory, and then moves the heads by 16 bytes a thread, several of them in flight.
#include <algorithm>
#include "ps_train.cuh"

namespace {
using namespace train;

constexpr int THREADS = 256, AT_ONCE = 4, TOKENS_MOST = 32;

__device__ __forceinline__ float2 turned(u64 turns, float magnitude) {
  const u64 quarter = (turns + ((u64)1 << 61)) >> 62;
  float s, c;
  sincospif((float)(s64)(turns - (quarter << 62)) * 0x1p-63f, &s, &c);
  const float2 v = quarter & 1 ? make_float2(-s, c) : make_float2(c, s);
  return quarter & 2 ? make_float2(-v.x * magnitude, -v.y * magnitude) : make_float2(v.x * magnitude, v.y * magnitude);
}

struct Plan {
  u32 tokens, a_block;          // all of them, and a block's
  u32 heads;                    // of q and k
  u32 items, turning;           // of a head: pairs of packs that turn (interleaved: packs), and packs that are copied
  Divider by_len, by_items, by_heads;
};

// N elements at a time.  (N = 1: elements or pairs at any alignment.)
template <class T, int N, bool INTERLEAVED>
__global__ void __launch_bounds__(THREADS) k_rotary(const __grid_constant__ RotaryArgs a, const Plan plan) {
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
    const u64 turns = (u64)(position + a.first) * a.turns[pair];
    circle[i] = turned(a.inverse ? 0 - turns : turns, a.magnitude);
  }
  __syncthreads();
  constexpr int SECOND = INTERLEAVED && N > 1 ? 0 : N;        // elements of an item's second part
  const u32 items = count * plan.heads * plan.items;
  for (u32 first = threadIdx.x; first < items; first += THREADS * AT_ONCE) {
    Pack<T, N> x[AT_ONCE], y[AT_ONCE];
    T* to[AT_ONCE];
    u32 apart[AT_ONCE], at[AT_ONCE];                          // second part behind the first; where the angles lie
#pragma unroll
    for (int u = 0; u < AT_ONCE; ++u) {
      const u32 item = first + u * THREADS;
      to[u] = nullptr;
      if (item < items) {
        const u32 row = plan.by_items.of(item), p = item - row * plan.items;
        const u32 t = plan.by_heads.of(row), h = row - t * plan.heads, token = begin + t;
        const u32 b = plan.by_len.of(token), i = token - b * a.len;
        const bool key = h >= a.heads;
        const ps_heads& from = key ? a.k : a.q;
        const ps_heads& into = key ? a.k_out : a.q_out;
        const u32 head = key ? h - a.heads : h;
        u32 column;
        at[u] = ~0u;
        apart[u] = 0;
        if (p < plan.turning) {
          if (INTERLEAVED) {
            column = N > 1 ? p * N : 2 * p;
            apart[u] = 1;
            at[u] = t * a.pairs + column / 2;
          } else {
            column = p * N;
            apart[u] = a.pairs;
            at[u] = t * a.pairs + column;
          }
        } else {
          column = 2 * a.pairs + (p - plan.turning) * N;
        }
        const T* const x_at = (const T*)from.data + b * from.batch_stride + i * from.token_stride + head * from.head_stride + column;
        to[u] = (T*)into.data + b * into.batch_stride + i * into.token_stride + head * into.head_stride + column;
        x[u].load(x_at);
        if (SECOND && at[u] != ~0u) y[u].load(x_at + apart[u]);
      }
    }
#pragma unroll
    for (int u = 0; u < AT_ONCE; ++u) {
      if (to[u] == nullptr) continue;
      if (at[u] != ~0u) {
        float v[N], w[N];
        x[u].widen(v);
        if (SECOND) {
          y[u].widen(w);
#pragma unroll
          for (int e = 0; e < N; ++e) {
            const float2 cs = circle[at[u] + e];
            const float turned_v = v[e] * cs.x - w[e] * cs.y;
            w[e] = w[e] * cs.x + v[e] * cs.y;
            v[e] = turned_v;
          }
          y[u].narrow(w);
          y[u].store(to[u] + apart[u]);
        } else {
#pragma unroll
          for (int e = 0; e + 1 < N; e += 2) {
            const float2 cs = circle[at[u] + e / 2];
            const float turned_v = v[e] * cs.x - v[e + 1] * cs.y;
            v[e + 1] = v[e + 1] * cs.x + v[e] * cs.y;
            v[e] = turned_v;
          }
        }
        x[u].narrow(v);
      }
      x[u].store(to[u]);
    }
  }
}

template <class T, int N, bool INTERLEAVED>
cudaError_t rotary(RotaryArgs a, cudaStream_t stream) {
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
  plan.by_items = Divider(plan.items);
  plan.by_heads = Divider(plan.heads);
  const u64 a_token = (u64)plan.heads * plan.items;
  plan.a_block = (u32)std::min<u64>(TOKENS_MOST, std::max<u64>(1, THREADS * AT_ONCE / a_token));
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
cudaError_t rotary(const RotaryArgs& a, cudaStream_t stream) {
  constexpr u32 N = 16 / sizeof(T);
  const auto packs = [&](const ps_heads& h) {
    return reinterpret_cast<uintptr_t>(h.data) % 16 == 0 && h.batch_stride % N == 0 && h.token_stride % N == 0 && h.head_stride % N == 0;
  };
  const bool wide = a.dim % N == 0 && (a.interleaved ? 2 * a.pairs : a.pairs) % N == 0 && packs(a.q) && packs(a.q_out) &&
                    (a.kv_heads == 0 || (packs(a.k) && packs(a.k_out)));
  if (wide) return a.interleaved ? rotary<T, N, true>(a, stream) : rotary<T, N, false>(a, stream);
  return a.interleaved ? rotary<T, 1, true>(a, stream) : rotary<T, 1, false>(a, stream);
}

}  // namespace

cudaError_t launch_rotary(u32 dtype, const RotaryArgs& a, int, cudaStream_t stream) {
  if (dtype == PS_F32) return rotary<float>(a, stream);
  return dtype == PS_BF16 ? rotary<__nv_bfloat16>(a, stream) : rotary<__half>(a, stream);
}
