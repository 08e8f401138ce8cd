// Attention and its backward pass.
//
//   S = scale * Q K^T over the keys a query sees;  lse_i = log sum_j exp(S_ij);  O = exp(S - lse) V
//   delta_i = sum_d dO_id O_id;  P = exp(S - lse);  dS = P o (dO V^T - delta)
//   dQ = scale * dS K;  dK = scale * dS^T Q;  dV = P^T dO       (dK, dV over the query heads of a key head)
//
// Query i of a sequence of n queries and m keys sees key j < m, under the causal mask those with j <= i + m - n.
// A query that sees nothing has O = 0 and lse = -infinity, and no gradient.  Queries behind n and keys behind m are
// padding: nothing of theirs is used, and zeros are written for them.
//
// All products run on the tensor cores (ps_tensor.cuh) on tiles of 128 queries and 128 keys; the matrices between two
// products (P, dS) stay in tensor memory.  A block has a warp that copies tiles, one or two that start products, and two
// groups of four warps that take the exponentials.
//
// Exponents are taken to base 2: exp(S - lse) = 2^(c S' - lse log2 e) with S' = Q K^T and c = |scale| log2 e (a negative
// scale negates an operand of the product; c is at least 1e-30, so that what a mask sets to -infinity stays there).
//
// The backward pass is two kernels, one that owns keys (dK, dV) and one that owns queries (dQ).  That is seven products a
// tile pair instead of the five of a single pass, which would have to add dQ from many blocks in memory: in an order
// that changes from run to run, or with waits between blocks.  So every result has one order of its sums.
#include <atomic>
#include "ps_tensor.cuh"

namespace {
using namespace train;
using namespace tensor;

constexpr float MINUS_INF = -INFINITY;
constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;
constexpr int THREADS = 384;            // two groups of four warps, and one of the copying warp, the two that start products and an idle one
constexpr int COPY_WARP = 8, MMA_WARP = 9, MMA_WARP2 = 10;
// Registers of a thread: as launched, and as the third group gives to the others.  (Forward, 8192 queries, 32 heads of 64: 437 us with 208
// and 88, where the groups spill, 366 with 216 and 72; of 128: 453 with either, 588 with 224 and 56, where the products' warp
// does.  Backward, heads of 128: 1508 with 208, 1543 with 216.)
constexpr int LAUNCHED = 168;
template <int TAKEN> struct Registers {
  static constexpr int taken = TAKEN, left = 3 * LAUNCHED - 2 * TAKEN;
};
typedef Registers<216> ForwardRegisters;
typedef Registers<208> BackwardRegisters;
static_assert(THREADS * LAUNCHED <= 65536, "registers that the block has");

// what a kernel needs beside the maps of its operands
struct Args {
  ps_heads out, d_q, d_k, d_v;
  float* lse;
  const int *q_lens, *k_lens;
  int batch, q_len, k_len, heads, kv_heads, dim, causal;
  float scale, c;
  // the backward pass's rows: -lse log2 e (-infinity for a query without keys) and -delta, of every query head with q_len
  // rounded up to whole tiles; and for types with a small range the norms, see gradient_factor
  float *lse2, *delta;
  u32* norms;
  u32* rows_there;      // see publish_rows
  int padded;
  // few queries before many keys, or the other way: the long side is cut into chunks, a block each, whose results in 32 bits are
  // joined by another kernel
  float *parts, *part_lse;
  volatile u32* status;
};
struct Lengths {
  int n, m;
};
__device__ __forceinline__ Lengths lengths_of(const Args& a, int b) {
  return {a.q_lens ? max(0, min(a.q_lens[b], a.q_len)) : a.q_len, a.k_lens ? max(0, min(a.k_lens[b], a.k_len)) : a.k_len};
}
// the keys that query i sees are those before this one
__device__ __forceinline__ int end_of(const Args& a, Lengths l, int i) {
  return i >= l.n ? 0 : a.causal ? max(0, min(l.m, i + l.m - l.n + 1)) : l.m;
}
// the tiles of keys that the 128 queries from i on see
__device__ __forceinline__ int key_tiles(const Args& a, Lengths l, int i) {
  return i >= l.n ? 0 : (end_of(a, l, min(i + ROWS, l.n) - 1) + ROWS - 1) / ROWS;
}

// the first tile of queries that sees keys from j on
__device__ __forceinline__ int first_query_tile(const Args& a, Lengths l, int j) { return a.causal ? max(0, j - l.m + l.n) / ROWS : 0; }

// A block of few rows would walk a long axis alone: at up to FEW rows of one side and more than two chunks of the other, blocks take
// a chunk of CHUNK tiles each.  The rule looks at the two lengths alone, so that a sequence's bits do not depend on how many
// others there are.  (Without rows there is nothing to cut, and nothing to join.)
constexpr int FEW = 2 * ROWS, CHUNK = 16;
__host__ __device__ constexpr bool chunked(int rows, int along) { return rows > 0 && rows <= FEW && along > 2 * CHUNK * ROWS; }
__host__ __device__ constexpr int chunks_of(int along) { return (along + CHUNK * ROWS - 1) / (CHUNK * ROWS); }

// 32 columns of a row of results, times `by`, to memory; columns behind dim are not there
template <class T>
__device__ __forceinline__ void store32(T* row, const u32 (&v)[32], int column, int dim, float by) {
#pragma unroll
  for (int c = 0; c < 32; c += 8)
    if (column + c < dim) {
      uint4 w;
      w.x = pack<T>(__uint_as_float(v[c]) * by, __uint_as_float(v[c + 1]) * by);
      w.y = pack<T>(__uint_as_float(v[c + 2]) * by, __uint_as_float(v[c + 3]) * by);
      w.z = pack<T>(__uint_as_float(v[c + 4]) * by, __uint_as_float(v[c + 5]) * by);
      w.w = pack<T>(__uint_as_float(v[c + 6]) * by, __uint_as_float(v[c + 7]) * by);
      *reinterpret_cast<uint4*>(row + column + c) = w;
    }
}
template <class T>
__device__ __forceinline__ T* row_of(const ps_heads& h, int b, int t, int head) {
  return (T*)h.data + b * h.batch_stride + t * h.token_stride + head * h.head_stride;
}
// a row of results from tensor memory (all lanes of a warp take part), or zeros
template <class T, int D>
__device__ __forceinline__ void store_row(T* row, u32 from, bool any, bool there, int dim, float by) {
#pragma unroll
  for (int c = 0; c < D; c += 32) {
    u32 v[32];
    if (any) {
      tmem_load32(v, from + c);
      wait_loads();
    }
    if (!any || by == 0.f)
#pragma unroll
      for (int e = 0; e < 32; ++e) v[e] = 0;
    if (there) store32(row, v, c, dim, by);
  }
}

// A block of the backward pass without work (its queries or keys are padding, or see nothing) leaves zeros and nothing else: it sets up
// no barriers and takes no tensor memory.  (Six sequences of 528 to 1475 padded to 2047, a half of the blocks: 193 us to 180.  In the forward pass
// it gained 2 us of 60 there and cost whole sequences with heads of 64 more.)
template <class T>
__device__ __forceinline__ void clear_results(const ps_heads& h, int b, int head, int first, int rows, int len, int dim) {
  const int packs = dim / 8, n = max(0, min(rows, len - first)) * packs;
  for (int i = threadIdx.x; i < n; i += blockDim.x) {
    const int r = i / packs;
    *reinterpret_cast<uint4*>(row_of<T>(h, b, first + r, head) + (i - r * packs) * 8) = make_uint4(0, 0, 0, 0);
  }
}

// a row of results in 32 bits, all D columns
template <int D>
__device__ __forceinline__ void store_part(float* row, u32 from, bool there, float by) {
#pragma unroll
  for (int c = 0; c < D; c += 32) {
    u32 v[32];
    tmem_load32(v, from + c);
    wait_loads();
    if (there)
#pragma unroll
      for (int e = 0; e < 32; e += 4)
        *reinterpret_cast<float4*>(row + c + e) = make_float4(__uint_as_float(v[e]) * by, __uint_as_float(v[e + 1]) * by,
                                                              __uint_as_float(v[e + 2]) * by, __uint_as_float(v[e + 3]) * by);
  }
}

// the smallest address in the block's shared memory that a tile may have
__device__ __forceinline__ u32 tiles_begin() {
  extern __shared__ unsigned char shared[];
  return (smem_address(shared) + 1023u) & ~1023u;
}
// leaving after a wait that did not end: copies and products that are still under way have time to end
__device__ __forceinline__ void linger(bool dead) {
  if (dead)
    for (int i = 0; i < 20; ++i) __nanosleep(1000000);
}

// Half precision has 2^-24 as its smallest number, and probabilities and gradients go below it.  P is held larger there, by
// 2^FORWARD_SHIFT in the forward pass and 2^P_SHIFT in the backward pass.  bfloat16 has float's exponents and needs nothing of the kind.
template <class T> struct Range { static constexpr bool small = false; };
template <> struct Range<__half> { static constexpr bool small = true; };
constexpr int FORWARD_SHIFT = 7, P_SHIFT = 12;

// ------------------------------------------------------------------ forward
// A block owns two tiles of 128 queries of a head, a group of warps each, a thread a query.  While one group takes the
// exponentials of its scores the tensor cores work for the other.  A group's turn: the scores S = Q K^T (128 columns of
// tensor memory), their row maximum, P = 2^(c S - c maximum) written over S in 16 bits, O += P V, begun when half of P is there.
// O is rescaled only when a row's maximum has grown by more than a factor of 2^8: until then P is larger than 1 by up
// to that, which the 32-bit sums and the types' exponents hold, and lse comes from the same maximum.
//
// In half precision P and its sum are both held 2^7 times as large, which with the 2^8 just fits: a probability keeps its 11 bits down to
// 2^-21 of the row's largest and is lost below 2^-32 of it; as it is, 2^-14 and 2^-25.  (2000 keys 14 below a key whose value is zero: out
// is off by 3.5e-3 as it is, and by its rounding with this; 16.5 below: 0.13 and 3e-3.  A factor of 2^9 leaves 2^6 until O is rescaled: 412 us instead
// of 391 with 8192 queries, 32 heads of 64 and scores of deviation 3; of 2^12 leaves 2^3: 426.)  Not so for scores of 2^20 and more, to
// base 2: the exponent of the largest is then off by as much as float32 rounds it, which would take P out of the type earlier.
//
// A product that writes tensor memory waits for the end of the one that reads it (S over P): nothing else orders products with
// different sums.  What bounds it, 8192 queries, 32 heads of 128 on 8 key heads, causal: 453 us, 1.21 PFLOP/s, the
// tensor pipe busy for 62 % and the special functions (16384 exponentials a tile pair, 16 a cycle) for 58 %, a group's chain S, exponentials,
// P V in between; after a second of it the power limit, 517 us.  Tried and slower: scores of 64 keys in two buffers (573: with 64
// columns a product is bound by shared memory), a warp for each tile's products (559: they interleave and both end late),
// a fourth of the exponentials as polynomials (448 against 440 then), blocks that take over others' work (registers).
template <class T, int D, bool CHUNKED>
__global__ void __launch_bounds__(THREADS, 1)
k_forward(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k,
          const __grid_constant__ CUtensorMap map_v, const Args a) {
  constexpr u32 TILE = PANEL * (D / 64);
  constexpr int RING = 4;
  constexpr bool TMEM = D == 64;          // Q is the left operand from tensor memory where there is room for it
  __shared__ u64 bars[2 + 2 * RING + 10];
  __shared__ u32 tmem_at;
  const u32 tiles = tiles_begin(), ring = tiles + 2 * TILE;
  const u32 q_full = smem_address(bars), full = q_full + 16, empty = full + 8 * RING, s_full = empty + 8 * RING,
            p_ready = s_full + 16, o_done = p_ready + 32, in_tmem = o_done + 16;
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;

  // the tiles with the most keys first
  const int per = a.heads * a.batch, n_tiles = (a.q_len + 2 * ROWS - 1) / (2 * ROWS), at = blockIdx.x / per;
  const int q0 = (a.causal ? n_tiles - 1 - at : at) * 2 * ROWS, b = blockIdx.x % per / a.heads, h = blockIdx.x % a.heads;
  const int kh = h / (a.heads / a.kv_heads);
  const Lengths l = lengths_of(a, b);
  const int skip = CHUNKED ? blockIdx.y * CHUNK : 0, key0 = skip * ROWS;        // tiles of keys before this block's, and its first key
  const auto tiles_of = [&](int i) { return CHUNKED ? max(0, min(key_tiles(a, l, i) - skip, CHUNK)) : key_tiles(a, l, i); };
  const int count0 = tiles_of(q0), count1 = tiles_of(q0 + ROWS), most = max(count0, count1);

  if (warp == MMA_WARP) tmem_alloc(smem_address(&tmem_at), 512);
  if (threadIdx.x == 0) {
    for (int t = 0; t < 2; ++t) {
      barrier_init(q_full + 8 * t, 1);
      barrier_init(s_full + 8 * t, 1);
      barrier_init(p_ready + 16 * t, 4);
      barrier_init(p_ready + 16 * t + 8, 4);
      barrier_init(o_done + 8 * t, 1);
      barrier_init(in_tmem + 8 * t, 4);
    }
    for (int i = 0; i < RING; ++i) {
      barrier_init(full + 8 * i, 1);
      barrier_init(empty + 8 * i, 1);
    }
    fence_barrier_init();
  }
  fence_before();
  __syncthreads();
  fence_after();
  const u32 tmem = tmem_at, tmem_q = tmem + 2 * ROWS + 2 * D;      // (D = 64)
  Waiter w(a.status);

  if (warp < COPY_WARP) {
    take_registers<ForwardRegisters::taken>();
    const int t = warp / 4, row = threadIdx.x % ROWS, i = q0 + t * ROWS + row, end = end_of(a, l, i) - key0;
    const u32 lanes = (u32)(warp % 4 * 32) << 16, s_at = tmem + lanes + t * ROWS, o_at = tmem + lanes + 2 * ROWS + t * D;
    // the first tile of keys of which some query of this tile does not see all
    const int masked = q0 + (t + 1) * ROWS > l.n ? 0 : (end_of(a, l, q0 + t * ROWS) - key0) / ROWS;
    const float slack = 8.f / a.c;
    // the power of two that P is held larger by, for a reference score
    const auto shift_of = [&](float most) { return Range<T>::small && fabsf(most * a.c) < 0x1p20f ? (float)FORWARD_SHIFT : 0.f; };
    const int count = t ? count1 : count0;
    float most_s = MINUS_INF, total = 0.f;
    if (TMEM && count) {
      w.wait(q_full + 8 * t, 0);
      tile_to_tmem<D>(tmem_q + lanes + t * (D / 2), tiles + t * TILE);
      if (lane == 0) barrier_arrive(in_tmem + 8 * t);
    }
    for (int j = 0; j < count; ++j) {
      w.wait(s_full + 8 * t, j & 1);
      fence_after();
      u32 s[4][32];
#pragma unroll
      for (int q = 0; q < 4; ++q) tmem_load32(s[q], s_at + 32 * q);
      wait_loads();
      if (j >= masked) {
        const int left = end - j * ROWS;
#pragma unroll
        for (int q = 0; q < 4; ++q)
#pragma unroll
          for (int e = 0; e < 32; ++e)
            if (32 * q + e >= left) s[q][e] = __float_as_uint(MINUS_INF);
      }
      float top[4] = {MINUS_INF, MINUS_INF, MINUS_INF, MINUS_INF};
#pragma unroll
      for (int e = 0; e < 32; ++e)
#pragma unroll
        for (int q = 0; q < 4; ++q) top[q] = fmaxf(top[q], __uint_as_float(s[q][e]));
      const float now = fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3]));
      const bool grown = now > most_s + slack;
      if (__any_sync(0xffffffffu, grown)) {
        const float by = grown ? exp2_fast((most_s - now) * a.c + (shift_of(now) - shift_of(most_s))) : 1.f;
        if (grown) most_s = now;
        total *= by;
        if (j > 0) {           // (the product that wrote O last is done: S, which was started behind its end, is there)
#pragma unroll
          for (int c = 0; c < D; c += 32) {
            u32 o[32];
            tmem_load32(o, o_at + c);
            wait_loads();
#pragma unroll
            for (int e = 0; e < 32; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * by);
            tmem_store32(o_at + c, o);
          }
        }
      }
      const float off = most_s == MINUS_INF ? 0.f : fmaf(-most_s, a.c, shift_of(most_s));
      const u64 offs = pair(off, off), cs = pair(a.c, a.c);
      u64 sum[2] = {0, 0};
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        u32 p[16];
#pragma unroll
        for (int e = 0; e < 32; e += 2) {
          const float2 x = exp2_pair(s[q][e], s[q][e + 1], cs, offs);
          sum[e / 2 & 1] = add2(sum[e / 2 & 1], pair(x.x, x.y));
          p[e / 2] = pack<T>(x.x, x.y);
        }
        tmem_store16(s_at + 16 * q, p);
        if (q & 1) {             // half of P: the product's first steps may begin
          wait_stores();
          fence_before();
          __syncwarp();
          if (lane == 0) barrier_arrive(p_ready + 16 * t + 8 * (q / 2));
        }
      }
      const float2 sums = split(add2(sum[0], sum[1]));
      total += sums.x + sums.y;
    }
    if (count) {
      w.wait(o_done + 8 * t, (count - 1) & 1);
      fence_after();
    }
    const bool there = i < a.q_len, none = most_s == MINUS_INF && total == 0.f;
    const int safe = min(i, a.q_len - 1);
    const float lse = none ? MINUS_INF : (most_s * a.c + log2f(Range<T>::small ? total * exp2_fast(-shift_of(most_s)) : total)) * LN2,
                by = none ? 0.f : 1.f / total;
    if constexpr (CHUNKED) {
      const u64 at = (((u64)blockIdx.y * a.batch + b) * a.heads + h) * a.q_len + safe;
      if (count) store_part<D>(a.parts + at * D, o_at, there, by);
      if (there) a.part_lse[at] = lse;
    } else {
      store_row<T, D>(row_of<T>(a.out, b, safe, h), o_at, count > 0, there, a.dim, by);
      if (there) a.lse[((u64)b * a.heads + h) * a.q_len + i] = lse;
    }
  } else if (warp == COPY_WARP) {
    give_registers<ForwardRegisters::left>();
    if (lane == 0) {
#pragma unroll
      for (int t = 0; t < 2; ++t)
        if (t ? count1 : count0) {
          barrier_expect(q_full + 8 * t, TILE);
          load_tile<D>(tiles + t * TILE, &map_q, h, q0 + t * ROWS, b, q_full + 8 * t);
        }
      for (int x = 0; x < 2 * most && !w.dead; ++x) {        // K of tile 0, V of tile 0, K of tile 1, ...
        const int slot = x % RING;
        w.wait(empty + 8 * slot, (x / RING & 1) ^ 1);
        if (w.dead) break;
        barrier_expect(full + 8 * slot, TILE);
        load_tile<D>(ring + slot * TILE, x & 1 ? &map_v : &map_k, kh, key0 + x / 2 * ROWS, b, full + 8 * slot);
      }
    }
  } else if (warp == MMA_WARP) {
    give_registers<ForwardRegisters::left>();
    const u32 ins_s = instruction<T>(ROWS, false, a.scale < 0), ins_o = instruction<T>(D, true, false);
    auto scores = [&](int t, int j) {
      const u32 k = ring + (2 * j % RING) * TILE;
      if (TMEM) multiply_along_tmem<D>(tmem + t * ROWS, tmem_q + t * (D / 2), k, ins_s);
      else multiply_along<D>(tmem + t * ROWS, tiles + t * TILE, k, ins_s);
      commit(s_full + 8 * t);
    };
    if (most > 0) {
      w.wait(full, 0);
#pragma unroll
      for (int t = 0; t < 2; ++t)
        if (t ? count1 : count0) {
          w.wait((TMEM ? in_tmem : q_full) + 8 * t, 0);
          fence_after();
          if (elected() && !w.dead) scores(t, 0);
        }
      if (elected() && !w.dead) commit(empty);
    }
    for (int j = 0; j < most; ++j) {
      const int x = 2 * j + 1, slot = x % RING, next = (x + 1) % RING;
      const u32 v = ring + slot * TILE;
      w.wait(full + 8 * slot, x / RING & 1);
      if (l.m < a.k_len && key0 + (j + 1) * ROWS > l.m) clear_rows<D>(v, l.m - key0 - j * ROWS);
      if (j + 1 < most) w.wait(full + 8 * next, (x + 1) / RING & 1);
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const int count = t ? count1 : count0;
        if (j >= count) continue;
#pragma unroll
        for (int part = 0; part < 2; ++part) {
          w.wait(p_ready + 16 * t + 8 * part, j & 1);
          fence_after();
          if (elected() && !w.dead) {
            multiply_across<ROWS / 2>(tmem + 2 * ROWS + t * D, tmem + t * ROWS + part * (ROWS / 4), v + part * (ROWS / 2) * 128, ins_o,
                                      j > 0 || part > 0);
            if (part) commit(o_done + 8 * t);
          }
          __syncwarp();
        }
        if (j + 1 < count) {           // S goes over P, which that product reads: nothing but its end orders the two
          w.wait(o_done + 8 * t, j & 1);
          fence_after();
          if (elected() && !w.dead) scores(t, j + 1);
          __syncwarp();
        }
      }
      if (elected() && !w.dead) {
        commit(empty + 8 * slot);
        if (j + 1 < most) commit(empty + 8 * next);
      }
      __syncwarp();
    }
  } else {
    give_registers<ForwardRegisters::left>();
  }
  linger(w.dead);
  fence_before();
  __syncthreads();
  if (warp == MMA_WARP) {
    fence_after();
    tmem_free(tmem, 512);
  }
}

// The chunks' outputs, each normalised by itself, weighted by exp(their lse - the row's): a warp a query.
template <class T, int D>
__global__ void __launch_bounds__(256) k_join_outputs(const Args a, int chunks) {
  wait_for_earlier();
  const int lane = threadIdx.x % 32, i = blockIdx.x * 8 + threadIdx.x / 32, h = blockIdx.y, b = blockIdx.z;
  if (i >= a.q_len) return;
  const u64 row = ((u64)b * a.heads + h) * a.q_len + i, stride = (u64)a.batch * a.heads * a.q_len;
  float most = MINUS_INF, total = 0.f, sum[D / 32] = {};
  for (int s = 0; s < chunks; ++s) most = fmaxf(most, a.part_lse[s * stride + row]);
  for (int s = 0; s < chunks; ++s) {
    const float lse = a.part_lse[s * stride + row];
    if (lse == MINUS_INF) continue;                  // (its output was not written)
    const float weight = exp2_fast((lse - most) * LOG2E);
    total += weight;
#pragma unroll
    for (int e = 0; e < D / 32; ++e) sum[e] = fmaf(weight, a.parts[(s * stride + row) * D + lane + 32 * e], sum[e]);
  }
  const float by = total > 0.f || total != total ? 1.f / total : 0.f;
  T* const to = row_of<T>(a.out, b, i, h);
#pragma unroll
  for (int e = 0; e < D / 32; ++e)
    if (lane + 32 * e < a.dim) to[lane + 32 * e] = narrow<T>(sum[e] * by);
  if (lane == 0) a.lse[row] = by == 0.f ? MINUS_INF : most + log2f(total) * LN2;
}

// ------------------------------------------------------------------ backward
// In half precision P is at most 2^P_SHIFT here, and dS is held times a power of two that follows from the largest norms: |dP - delta| is at
// most 2 |dO_i| |V_j|, and that bound is brought to 2^14 or just below for each key head (its queries are summed over).
// dS is held times 2^P_SHIFT times this
__device__ __forceinline__ float gradient_factor(const Args& a, int b, int kh) {
  const u32* at = a.norms + 2 * (b * a.kv_heads + kh);
  const float bound = 2.f * sqrtf(__uint_as_float(at[0])) * sqrtf(__uint_as_float(at[1]));
  if (!(bound > 0.f && bound < INFINITY)) return exp2_fast(-P_SHIFT);
  const int e = 14 - ilogbf(bound) - 1;
  return exp2_fast((float)(max(-60, min(60, e)) - P_SHIFT));
}

// The rows that both kernels read: D / 8 lanes a query, delta and the exponent's offset; in half precision the largest
// norms of each key head's dO and V rows as well (as bits: norms are not negative, so they compare as integers), one atomic
// a block.
constexpr int ROWS_A_THREAD = 4;
template <int D> constexpr int ROWS_A_BLOCK = 256 / (D / 8) * ROWS_A_THREAD;
template <class T, int D, bool QUERY>
__global__ void __launch_bounds__(256) k_rows(const ps_heads x, const ps_heads out, const Args a) {
  let_next_begin();
  if (QUERY && (threadIdx.x | blockIdx.x | blockIdx.y | blockIdx.z) == 0) *a.rows_there = 0;
  __shared__ u32 largest;
  if (Range<T>::small) {
    if (threadIdx.x == 0) largest = 0;
    __syncthreads();
  }
  constexpr int LANES = D / 8, STEP = 256 / LANES;
  const int part = threadIdx.x % LANES, first = blockIdx.x * ROWS_A_BLOCK<D> + threadIdx.x / LANES, h = blockIdx.y, b = blockIdx.z;
  const Lengths l = lengths_of(a, b);
  Pack<T, 8> p[ROWS_A_THREAD], q[ROWS_A_THREAD];
#pragma unroll
  for (int r = 0; r < ROWS_A_THREAD; ++r) {
    const int i = first + STEP * r;
    p[r].clear();
    q[r].clear();
    if (i < (QUERY ? l.n : l.m) && part * 8 < a.dim) {
      p[r].load(row_of<const T>(x, b, i, h) + part * 8);
      if (QUERY) q[r].load(row_of<const T>(out, b, i, h) + part * 8);
    }
  }
#pragma unroll
  for (int r = 0; r < ROWS_A_THREAD; ++r) {
    const int i = first + STEP * r;
    float v[8], y[8], dot = 0.f, norm = 0.f;
    p[r].widen(v);
    q[r].widen(y);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      if (QUERY) dot = fmaf(v[e], y[e], dot);
      if (Range<T>::small) norm = fmaf(v[e], v[e], norm);
    }
#pragma unroll
    for (int o = LANES / 2; o > 0; o >>= 1) {
      if (QUERY) dot += __shfl_xor_sync(0xffffffffu, dot, o);
      if (Range<T>::small) norm += __shfl_xor_sync(0xffffffffu, norm, o);
    }
    if (part != 0 || i >= (QUERY ? a.padded : a.k_len)) continue;
    if (QUERY) {
      const u64 head = (u64)b * a.heads + h;
      const float lse = i < l.n ? a.lse[head * a.q_len + i] : MINUS_INF;
      a.lse2[head * a.padded + i] = lse == MINUS_INF || end_of(a, l, i) == 0 ? MINUS_INF : (Range<T>::small ? P_SHIFT : 0) - lse * LOG2E;
      a.delta[head * a.padded + i] = -dot;
    }
    if (Range<T>::small) atomicMax(&largest, __float_as_uint(norm));
  }
  if (Range<T>::small) {
    __syncthreads();
    if (threadIdx.x == 0) atomicMax(a.norms + 2 * (b * a.kv_heads + (QUERY ? h / (a.heads / a.kv_heads) : h)) + (QUERY ? 0 : 1), largest);
  }
}

// k_queries may begin while k_keys runs, and reads what k_rows wrote: the kernel before the one that its wait is for.  So a thread of each
// block of k_keys, behind that block's wait for the rows, says so in memory before it lets k_queries begin, and whoever reads that there
// sees the rows as well.  Else k_queries waits for all of k_keys.
__device__ __forceinline__ void publish_rows(const Args& a) {
  asm volatile("st.release.gpu.global.u32 [%0], %1;" ::"l"(a.rows_there), "r"(1u) : "memory");
}
__device__ __forceinline__ void wait_for_rows(const Args& a) {
  u32 there;
  asm volatile("ld.acquire.gpu.global.u32 %0, [%1];" : "=r"(there) : "l"(a.rows_there) : "memory");
  if (!there) wait_for_earlier();
}

// Both kernels of the backward pass let their two groups of warps take turns: tile pairs are numbered, a group has the even
// ones and the other the odd ones, each with a buffer of 128 columns of tensor memory of its own, a thread a row.  A
// pair's buffer holds S, then what its products leave of P, then dP, then dS.  While one group works the tensor cores
// multiply for the other.  One warp starts the products that add to the results, in the pairs' order, and another those that
// fill the buffers, each behind the end of the product that reads what it overwrites (one warp for both: 1577 us for the case below
// instead of 1512; both groups on each pair, a half of it each: 2008).
//
// Shared memory is full (224 KB of tiles for D = 128), so barriers and vectors share what is behind the tiles.
struct Shared {
  u64 bars[24];
  u32 tmem_at;
};

// A block owns 128 keys of a key head and walks the queries that see them, through all query heads that share it.  Scores are
// transposed: S^T = K Q^T has a key a lane, so P^T and dS^T are left operands in tensor memory, and Q and dO serve as right
// operands of both kinds from one copy.  Tensor memory (D = 128): the two buffers, dV and dK, 128 columns each.
// Q has three slots, since S of pair x + 2 follows on dK of pair x; dO, with two, is free after dP.
// With D = 64 there is room for dP apart from the buffers, where P then lies beside dS: dP is multiplied during the exponentials and not
// behind dV, which takes a pair from 2544 to 2304 cycles (8192 queries, 32 heads on 8, causal; the whole pass 1214 us to 1112, or 1312 to 1209 on
// a warmer GPU), although K and V are read from shared memory for it, which slows the other group's exponentials.
// What bounds it, 8192 queries, 32 heads of 128 on 8 key heads, causal: 0.88 ms, the tensor pipe busy for 69 %: S and dP take both
// operands from shared memory, whose 128 bytes a cycle they use up, and the rest is the chain of a pair.
template <class T, int D, bool CHUNKED>
__global__ void __launch_bounds__(THREADS, 1)
k_keys(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k,
       const __grid_constant__ CUtensorMap map_v, const __grid_constant__ CUtensorMap map_do, const Args a) {
  constexpr u32 TILE = PANEL * (D / 64), VECTOR = ROWS * 4;
  constexpr bool APART = D == 64;         // dP has columns of its own
  extern __shared__ __align__(1024) unsigned char shared[];
  const u32 k_tile = smem_address(shared), v_tile = k_tile + TILE, q_ring = v_tile + TILE, do_ring = q_ring + 3 * TILE,
            lse_ring = do_ring + 2 * TILE, delta_ring = lse_ring + 3 * VECTOR;
  Shared& sh = *reinterpret_cast<Shared*>(shared + 7 * TILE + 5 * VECTOR);
  const u32 kv_full = smem_address(sh.bars), q_full = kv_full + 8, q_empty = q_full + 24, do_full = q_empty + 24, do_empty = do_full + 16,
            delta_full = do_empty + 16, s_full = delta_full + 16, p_ready = s_full + 16, dp_full = p_ready + 16,
            ds_ready = dp_full + 16, done = ds_ready + 16, dv_done = done + 8;
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;

  // (under the causal mask the first keys have the most queries)
  const int per = a.kv_heads * a.batch, j0 = blockIdx.x / per * ROWS, b = blockIdx.x % per / a.kv_heads, kh = blockIdx.x % a.kv_heads;
  const int group = a.heads / a.kv_heads;
  const Lengths l = lengths_of(a, b);
  const int first = first_query_tile(a, l, j0) + (CHUNKED ? blockIdx.y * CHUNK : 0), rest = (l.n + ROWS - 1) / ROWS - first;
  const int walk = j0 < l.m ? max(0, CHUNKED ? min(rest, CHUNK) : rest) : 0, total = walk * group;     // tiles of queries
  if (total == 0) {
    wait_for_earlier();
    if (threadIdx.x == 0) {
      publish_rows(a);
      let_next_begin();
    }
    if (!CHUNKED) {
      clear_results<T>(a.d_v, b, kh, j0, ROWS, a.k_len, a.dim);
      clear_results<T>(a.d_k, b, kh, j0, ROWS, a.k_len, a.dim);
    }
    return;
  }

  if (warp == MMA_WARP) tmem_alloc(smem_address(&sh.tmem_at), 512);
  if (threadIdx.x == 0) {
    barrier_init(kv_full, 1);
    for (int i = 0; i < 3; ++i) {
      barrier_init(q_full + 8 * i, 1);
      barrier_init(q_empty + 8 * i, 1);
    }
    for (int i = 0; i < 2; ++i) {
      barrier_init(do_full + 8 * i, 1);
      barrier_init(do_empty + 8 * i, 1);
      barrier_init(delta_full + 8 * i, 1);
      barrier_init(s_full + 8 * i, 1);
      barrier_init(p_ready + 8 * i, 4);
      barrier_init(dp_full + 8 * i, 1);
      barrier_init(ds_ready + 8 * i, 4);
      barrier_init(dv_done + 8 * i, 1);
    }
    barrier_init(done, 1);
    fence_barrier_init();
  }
  fence_before();
  __syncthreads();
  fence_after();
  // columns: the two buffers, dP where it is apart, dV, dK
  const u32 tmem = sh.tmem_at, tmem_dp = tmem + 2 * ROWS, tmem_dv = tmem + (APART ? 3 : 2) * ROWS, tmem_dk = tmem_dv + D;
  Waiter w(a.status);

  if (warp < COPY_WARP) {
    take_registers<BackwardRegisters::taken>();
    wait_for_earlier();          // the rows
    if (threadIdx.x == 0) {
      publish_rows(a);
      let_next_begin();          // k_queries needs the rows too, and nothing of this kernel
    }
    const int mine = warp / 4, j = j0 + threadIdx.x % ROWS;
    const u32 lanes = (u32)(warp % 4 * 32) << 16, at = tmem + lanes + mine * ROWS;
    // this key's first query; the first query that all of the tile's keys have
    const int begin = j >= l.m ? 0x7fffffff : a.causal ? j - l.m + l.n : 0;
    const int whole = j0 + ROWS > l.m ? 0x7fffffff : a.causal ? j0 + ROWS - 1 - l.m + l.n : 0;
    const float factor = Range<T>::small ? gradient_factor(a, b, kh) : 1.f;
    const u64 cs = pair(a.c, a.c), factors = pair(factor, factor);
    const u32 dp_at = APART ? tmem_dp + lanes : at, ds_at = APART ? at + ROWS / 2 : at;      // (P takes half of a buffer)
    for (int x = mine; x < total; x += 2) {
      const int i0 = (first + x % walk) * ROWS, turn = x >> 1 & 1;
      const float4* const lse_at = reinterpret_cast<const float4*>(shared + 7 * TILE + x % 3 * VECTOR);
      const float4* const delta_at = reinterpret_cast<const float4*>(shared + 7 * TILE + (3 + mine) * VECTOR);
      w.wait(q_full + 8 * (x % 3), x / 3 & 1);
      w.wait(s_full + 8 * mine, turn);
      fence_after();
      u32 p[4][32];
#pragma unroll
      for (int q = 0; q < 4; ++q) tmem_load32(p[q], at + 32 * q);
      wait_loads();
#pragma unroll
      for (int q = 0; q < 4; ++q) {
#pragma unroll
        for (int e = 0; e < 32; e += 4) {
          const float4 o = lse_at[(32 * q + e) / 4];
          const u64 off[2] = {pair(o.x, o.y), pair(o.z, o.w)};
#pragma unroll
          for (int f = 0; f < 4; f += 2) {
            const float2 y = exp2_pair(p[q][e + f], p[q][e + f + 1], cs, off[f / 2]);
            p[q][e + f] = __float_as_uint(y.x);
            p[q][e + f + 1] = __float_as_uint(y.y);
          }
        }
        if (i0 < whole) {
          const int skip = begin - i0 - 32 * q;
#pragma unroll
          for (int e = 0; e < 32; ++e)
            if (e < skip) p[q][e] = 0;
        }
        u32 out[16];
#pragma unroll
        for (int e = 0; e < 16; ++e) out[e] = pack<T>(__uint_as_float(p[q][2 * e]), __uint_as_float(p[q][2 * e + 1]));
        tmem_store16(at + 16 * q, out);
      }
      wait_stores();
      fence_before();
      __syncwarp();
      if (lane == 0) barrier_arrive(p_ready + 8 * mine);
      w.wait(delta_full + 8 * mine, turn);
      w.wait(dp_full + 8 * mine, turn);
      fence_after();
      u32 d[2][16];
      tmem_load16(d[0], dp_at);
      wait_loads();
#pragma unroll
      for (int q = 0; q < 8; ++q) {
        if (q < 7) tmem_load16(d[(q + 1) & 1], dp_at + 16 * (q + 1));
        u32 out[8];
#pragma unroll
        for (int e = 0; e < 16; e += 4) {
          const float4 o = delta_at[(16 * q + e) / 4];
          const u64 off[2] = {pair(o.x, o.y), pair(o.z, o.w)};
#pragma unroll
          for (int f = 0; f < 4; f += 2) {
            const int c = 16 * (q & 1) + e + f;
            u64 u = add2(pair(__uint_as_float(d[q & 1][e + f]), __uint_as_float(d[q & 1][e + f + 1])), off[f / 2]);
            if (Range<T>::small) u = mul2(u, factors);
            const float2 y = split(mul2(u, pair(__uint_as_float(p[q / 2][c]), __uint_as_float(p[q / 2][c + 1]))));
            out[(e + f) / 2] = pack<T>(y.x, y.y);
          }
        }
        wait_loads();                // (dS goes over columns that have been read)
        tmem_store8(ds_at + 8 * q, out);
      }
      wait_stores();
      fence_before();
      __syncwarp();
      if (lane == 0) barrier_arrive(ds_ready + 8 * mine);
    }
    w.wait(done, 0);
    fence_after();
    // one group stores dV, the other dK
    const bool there = j < a.k_len;
    const int safe = min(j, a.k_len - 1);
    const float undo = Range<T>::small ? exp2_fast(-P_SHIFT) : 1.f;
    const float by = mine ? a.scale / factor * undo : undo;
    const u32 from = (mine ? tmem_dk : tmem_dv) + lanes;
    if constexpr (CHUNKED) {
      store_part<D>(a.parts + ((((u64)(2 * blockIdx.y + mine) * a.batch + b) * a.kv_heads + kh) * a.k_len + safe) * D, from, there, by);
    } else {
      store_row<T, D>(row_of<T>(mine ? a.d_k : a.d_v, b, safe, kh), from, true, there, a.dim, j < l.m ? by : 0.f);
    }
  } else if (warp == COPY_WARP) {
    give_registers<BackwardRegisters::left>();
    if (lane == 0) {
      barrier_expect(kv_full, 2 * TILE);
      load_tile<D>(k_tile, &map_k, kh, j0, b, kv_full);
      load_tile<D>(v_tile, &map_v, kh, j0, b, kv_full);
      for (int x = 0; x < total; ++x) {
        const int slot = x % 3, two = x & 1, h = kh * group + x / walk, i0 = (first + x % walk) * ROWS;
        const u64 row = ((u64)b * a.heads + h) * a.padded + i0;
        w.wait(q_empty + 8 * slot, (x / 3 & 1) ^ 1);
        if (w.dead) break;
        barrier_expect(q_full + 8 * slot, TILE + VECTOR);
        load_tile<D>(q_ring + slot * TILE, &map_q, h, i0, b, q_full + 8 * slot);
        if (x == 0) wait_for_earlier();          // (tiles come from the caller, vectors from the rows' kernel)
        load_bytes(lse_ring + slot * VECTOR, a.lse2 + row, VECTOR, q_full + 8 * slot);
        w.wait(do_empty + 8 * two, (x >> 1 & 1) ^ 1);
        if (w.dead) break;
        barrier_expect(do_full + 8 * two, TILE);
        load_tile<D>(do_ring + two * TILE, &map_do, h, i0, b, do_full + 8 * two);
        // the delta before last has been read once its pair's dK is done
        if (x >= 2) w.wait(q_empty + 8 * ((x - 2) % 3), (x - 2) / 3 & 1);
        if (w.dead) break;
        barrier_expect(delta_full + 8 * two, VECTOR);
        load_bytes(delta_ring + two * VECTOR, a.delta + row, VECTOR, delta_full + 8 * two);
      }
    }
  } else if (warp == MMA_WARP || warp == MMA_WARP2) {
    // One warp starts the sums dV and dK, in the pairs' order, the other the products that fill the buffers.  A product that
    // writes a buffer waits for the end of the one that reads it: nothing else orders the two.
    give_registers<BackwardRegisters::left>();
    // queries behind the sequence's end, in its last tile
    auto pad_from = [&](int x) {
      const int i0 = (first + x % walk) * ROWS;
      return l.n < a.q_len && i0 + ROWS > l.n ? l.n - i0 : ROWS;
    };
    if (warp == MMA_WARP) {
      const u32 ins = instruction<T>(D, true, false);
      auto values = [&](int x) {                 // dV += P^T dO
        const int two = x & 1;
        const u32 d = do_ring + two * TILE;
        if (APART) {
          w.wait(dp_full + 8 * two, x >> 1 & 1);           // (dP has read dO before, and cleared what is behind the end)
        } else {
          w.wait(do_full + 8 * two, x >> 1 & 1);
          if (pad_from(x) < ROWS) clear_rows<D>(d, pad_from(x));
        }
        w.wait(p_ready + 8 * two, x >> 1 & 1);
        fence_after();
        if (elected() && !w.dead) {
          multiply_across(tmem_dv, tmem + two * ROWS, d, ins, x > 0);
          commit((APART ? do_empty : dv_done) + 8 * two);
        }
        __syncwarp();
      };
      auto keys = [&](int x) {                   // dK += dS^T Q
        const int two = x & 1;
        w.wait(ds_ready + 8 * two, x >> 1 & 1);
        fence_after();
        if (elected() && !w.dead) {
          multiply_across(tmem_dk, tmem + two * ROWS + (APART ? ROWS / 2 : 0), q_ring + x % 3 * TILE, ins, x > 0);
          commit(q_empty + 8 * (x % 3));
          if (x + 1 == total) commit(done);
        }
        __syncwarp();
      };
      if (APART) {
        for (int x = 0; x < total; ++x) {
          values(x);
          keys(x);
        }
      } else {
        for (int x = 0; x < total; x += 2) {
          values(x);
          if (x + 1 < total) values(x + 1);
          keys(x);
          if (x + 1 < total) keys(x + 1);
        }
      }
    } else {
      const u32 ins_s = instruction<T>(ROWS, false, a.scale < 0), ins_dp = instruction<T>(ROWS, false, false);
      auto scores = [&](int x) {                 // S^T = K Q^T, over dS^T of pair x - 2
        const u32 q = q_ring + x % 3 * TILE;
        w.wait(q_full + 8 * (x % 3), x / 3 & 1);
        if (pad_from(x) < ROWS) clear_rows<D>(q, pad_from(x));
        if (x >= 2) w.wait(q_empty + 8 * ((x - 2) % 3), (x - 2) / 3 & 1);
        fence_after();
        if (elected() && !w.dead) {
          multiply_along<D>(tmem + (x & 1) * ROWS, k_tile, q, ins_s);
          commit(s_full + 8 * (x & 1));
        }
        __syncwarp();
      };
      auto d_probabilities = [&](int x) {        // dP^T = V dO^T, over P^T or over dP^T of pair x - 1
        const int two = x & 1;
        const u32 d = do_ring + two * TILE;
        if (APART) {
          w.wait(do_full + 8 * two, x >> 1 & 1);
          if (pad_from(x) < ROWS) clear_rows<D>(d, pad_from(x));
          if (x > 0) w.wait(ds_ready + 8 * (two ^ 1), (x - 1) >> 1 & 1);
        } else {
          w.wait(dv_done + 8 * two, x >> 1 & 1);
        }
        fence_after();
        if (elected() && !w.dead) {
          multiply_along<D>(APART ? tmem_dp : tmem + two * ROWS, v_tile, d, ins_dp);
          commit(dp_full + 8 * two);
          if (!APART) commit(do_empty + 8 * two);
        }
        __syncwarp();
      };
      w.wait(kv_full, 0);
      fence_after();
      scores(0);
      if (total > 1) scores(1);
      if (APART) {
        d_probabilities(0);
        for (int x = 0; x < total; ++x) {
          if (x + 1 < total) d_probabilities(x + 1);
          if (x + 2 < total) scores(x + 2);
        }
      } else {
        for (int x = 0; x < total; x += 2) {
          d_probabilities(x);
          if (x + 1 < total) d_probabilities(x + 1);
          if (x + 2 < total) scores(x + 2);
          if (x + 3 < total) scores(x + 3);
        }
      }
    }
  } else {
    give_registers<BackwardRegisters::left>();
  }
  linger(w.dead);
  fence_before();
  __syncthreads();
  if (warp == MMA_WARP) {
    fence_after();
    tmem_free(tmem, 512);
  }
}

// With heads of up to 64 a block has one group, one buffer and half of the tensor memory, and an SM has two such blocks:
// they take turns like the groups of one, and one begins or ends while the other works.  (A block has 5 tiles of keys on average in six sequences
// of 528 to 1475, 16 heads: the whole pass 177 us with 192 and 64 registers, 188 with one block of two groups; 8192 queries with 32 heads 1104 and
// 1120.  184 registers spill in the group, and 200 leave too few to the warps that start products.)
template <int D> struct QueryBlock {
  static constexpr int groups = D == 64 ? 1 : 2, threads = 128 * (groups + 1), resident = 3 - groups, columns = 256 * groups;
  static constexpr int launched = groups == 1 ? 128 : LAUNCHED, taken = groups == 1 ? 192 : BackwardRegisters::taken,
                       left = (groups + 1) * launched - groups * taken;
  static_assert(resident * threads * launched <= 65536, "registers that the blocks have");
};

// A block owns 128 queries of a head and walks the keys they see.  P stays in registers, so dP may be written over S as soon as S
// has been read.  Tensor memory (D = 128): the two buffers, dQ, and Q and dO as left operands (from shared memory: 1512 us for the
// whole pass then, 1487 so).  K has three slots, V two, as Q and dO above.  The same case: 0.67 ms, the tensor pipe
// busy for 65 %.  A third buffer of scores, with Q and dO in shared memory again, took as long.
template <class T, int D, bool CHUNKED>
__global__ void __launch_bounds__(QueryBlock<D>::threads, QueryBlock<D>::resident)
k_queries(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k,
          const __grid_constant__ CUtensorMap map_v, const __grid_constant__ CUtensorMap map_do, const Args a) {
  constexpr u32 TILE = PANEL * (D / 64);
  typedef QueryBlock<D> Block;
  constexpr int GROUPS = Block::groups, COPY_WARP = 4 * GROUPS, MMA_WARP = COPY_WARP + 1, MMA_WARP2 = COPY_WARP + 2;
  extern __shared__ __align__(1024) unsigned char shared[];
  const u32 q_tile = smem_address(shared), do_tile = q_tile + TILE, k_ring = do_tile + TILE, v_ring = k_ring + 3 * TILE;
  Shared& sh = *reinterpret_cast<Shared*>(shared + 7 * TILE);
  const u32 q_full = smem_address(sh.bars), k_full = q_full + 8, k_empty = k_full + 24, v_full = k_empty + 24, v_empty = v_full + 16,
            s_full = v_empty + 16, s_read = s_full + 16, dp_full = s_read + 16, ds_ready = dp_full + 16, done = ds_ready + 16,
            in_tmem = done + 8;
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;

  const int per = a.heads * a.batch, n_tiles = (a.q_len + ROWS - 1) / ROWS, order = blockIdx.x / per;
  const int q0 = (a.causal ? n_tiles - 1 - order : order) * ROWS, b = blockIdx.x % per / a.heads, h = blockIdx.x % a.heads;
  const int kh = h / (a.heads / a.kv_heads);
  const Lengths l = lengths_of(a, b);
  const int skip = CHUNKED ? blockIdx.y * CHUNK : 0, key0 = skip * ROWS;        // tiles of keys before this block's, and its first key
  const int total = CHUNKED ? max(0, min(key_tiles(a, l, q0) - skip, CHUNK)) : key_tiles(a, l, q0);
  if (total == 0) {
    if (!CHUNKED) clear_results<T>(a.d_q, b, h, q0, ROWS, a.q_len, a.dim);
    wait_for_earlier();
    return;
  }

  if (warp == MMA_WARP) tmem_alloc(smem_address(&sh.tmem_at), Block::columns);
  if (threadIdx.x == 0) {
    barrier_init(q_full, 1);
    for (int i = 0; i < 3; ++i) {
      barrier_init(k_full + 8 * i, 1);
      barrier_init(k_empty + 8 * i, 1);
    }
    for (int i = 0; i < 2; ++i) {
      barrier_init(v_full + 8 * i, 1);
      barrier_init(v_empty + 8 * i, 1);
      barrier_init(s_full + 8 * i, 1);
      barrier_init(s_read + 8 * i, 4);
      barrier_init(dp_full + 8 * i, 1);
      barrier_init(ds_ready + 8 * i, 4);
    }
    barrier_init(done, 1);
    barrier_init(in_tmem, 4 * GROUPS);
    fence_barrier_init();
  }
  fence_before();
  __syncthreads();
  fence_after();
  const u32 tmem = sh.tmem_at, tmem_dq = tmem + GROUPS * ROWS, tmem_q = tmem_dq + D, tmem_do = tmem_q + D / 2;
  Waiter w(a.status);

  if (warp < COPY_WARP) {
    take_registers<Block::taken>();
    const int mine = warp / 4, i = q0 + threadIdx.x % ROWS, end = end_of(a, l, i) - key0;
    const u32 lanes = (u32)(warp % 4 * 32) << 16, at = tmem + lanes + mine * ROWS;
    const int masked = q0 + ROWS > l.n ? 0 : (end_of(a, l, q0) - key0) / ROWS;
    const u64 row = ((u64)b * a.heads + h) * a.padded + i;
    wait_for_rows(a);
    const float off = a.lse2[row], delta = a.delta[row], factor = Range<T>::small ? gradient_factor(a, b, kh) : 1.f;
    const u64 cs = pair(a.c, a.c), offs = pair(off, off), deltas = pair(delta, delta), factors = pair(factor, factor);
    w.wait(q_full, 0);          // Q and dO are left operands of every pair
    if (mine == 0) tile_to_tmem<D>(tmem_q + lanes, q_tile);
    if (mine == GROUPS - 1) tile_to_tmem<D>(tmem_do + lanes, do_tile);
    if (lane == 0) barrier_arrive(in_tmem);
    for (int x = mine; x < total; x += GROUPS) {
      const int turn = x / GROUPS & 1;
      w.wait(s_full + 8 * mine, turn);
      fence_after();
      u32 p[4][32];
#pragma unroll
      for (int q = 0; q < 4; ++q) tmem_load32(p[q], at + 32 * q);
      wait_loads();
      fence_before();
      __syncwarp();
      if (lane == 0) barrier_arrive(s_read + 8 * mine);
#pragma unroll
      for (int q = 0; q < 4; ++q) {
#pragma unroll
        for (int e = 0; e < 32; e += 2) {
          const float2 y = exp2_pair(p[q][e], p[q][e + 1], cs, offs);
          p[q][e] = __float_as_uint(y.x);
          p[q][e + 1] = __float_as_uint(y.y);
        }
        if (x >= masked) {
          const int left = end - x * ROWS - 32 * q;
#pragma unroll
          for (int e = 0; e < 32; ++e)
            if (e >= left) p[q][e] = 0;
        }
      }
      w.wait(dp_full + 8 * mine, turn);
      fence_after();
      u32 d[2][16];
      tmem_load16(d[0], at);
      wait_loads();
#pragma unroll
      for (int q = 0; q < 8; ++q) {
        if (q < 7) tmem_load16(d[(q + 1) & 1], at + 16 * (q + 1));
        u32 out[8];
#pragma unroll
        for (int e = 0; e < 16; e += 2) {
          const int c = 16 * (q & 1) + e;
          u64 u = add2(pair(__uint_as_float(d[q & 1][e]), __uint_as_float(d[q & 1][e + 1])), deltas);
          if (Range<T>::small) u = mul2(u, factors);
          const float2 y = split(mul2(u, pair(__uint_as_float(p[q / 2][c]), __uint_as_float(p[q / 2][c + 1]))));
          out[e / 2] = pack<T>(y.x, y.y);
        }
        wait_loads();                // (dS goes over columns that have been read)
        tmem_store8(at + 8 * q, out);
      }
      wait_stores();
      fence_before();
      __syncwarp();
      if (lane == 0) barrier_arrive(ds_ready + 8 * mine);
    }
    w.wait(done, 0);
    fence_after();
    // each group stores its share of the columns
    constexpr int SHARE = D / GROUPS;
    const bool there = i < a.q_len;
    const int safe = min(i, a.q_len - 1);
    const float by = off == MINUS_INF ? 0.f : a.scale / factor * (Range<T>::small ? exp2_fast(-P_SHIFT) : 1.f);
    const u32 from = tmem_dq + lanes + mine * SHARE;
    if constexpr (CHUNKED) {
      store_part<SHARE>(a.parts + ((((u64)blockIdx.y * a.batch + b) * a.heads + h) * a.q_len + safe) * D + mine * SHARE, from, there, by);
    } else {
      // (total is above 0.  With a constant in its place 8192 queries, 32 heads of 128 take 1583 us instead of 1555.)
      store_row<T, SHARE>(row_of<T>(a.d_q, b, safe, h) + mine * SHARE, from, total > 0, there, a.dim - mine * SHARE, by);
    }
  } else if (warp == COPY_WARP) {
    give_registers<Block::left>();
    if (lane == 0) {
      barrier_expect(q_full, 2 * TILE);
      load_tile<D>(q_tile, &map_q, h, q0, b, q_full);
      load_tile<D>(do_tile, &map_do, h, q0, b, q_full);
      for (int x = 0; x < total; ++x) {
        const int slot = x % 3, two = x & 1;
        w.wait(k_empty + 8 * slot, (x / 3 & 1) ^ 1);
        if (w.dead) break;
        barrier_expect(k_full + 8 * slot, TILE);
        load_tile<D>(k_ring + slot * TILE, &map_k, kh, key0 + x * ROWS, b, k_full + 8 * slot);
        w.wait(v_empty + 8 * two, (x >> 1 & 1) ^ 1);
        if (w.dead) break;
        barrier_expect(v_full + 8 * two, TILE);
        load_tile<D>(v_ring + two * TILE, &map_v, kh, key0 + x * ROWS, b, v_full + 8 * two);
      }
    }
  } else if (warp == MMA_WARP || warp == MMA_WARP2) {
    // (as in k_keys: one warp for the sum, the other for the products that fill the buffers)
    give_registers<Block::left>();
    if (warp == MMA_WARP) {
      const u32 ins = instruction<T>(D, true, false);
      for (int x = 0; x < total; ++x) {          // dQ += dS K
        const int at = x % GROUPS;
        w.wait(ds_ready + 8 * at, x / GROUPS & 1);
        fence_after();
        if (elected() && !w.dead) {
          multiply_across(tmem_dq, tmem + at * ROWS, k_ring + x % 3 * TILE, ins, x > 0);
          commit(k_empty + 8 * (x % 3));
          if (x + 1 == total) commit(done);
        }
        __syncwarp();
      }
    } else {
      const u32 ins_s = instruction<T>(ROWS, false, a.scale < 0), ins_dp = instruction<T>(ROWS, false, false);
      // keys behind the sequence's end, in its last tile
      auto pad_from = [&](int x) { return l.m < a.k_len && key0 + (x + 1) * ROWS > l.m ? l.m - key0 - x * ROWS : ROWS; };
      auto scores = [&](int x) {                 // S = Q K^T, over dS of pair x - GROUPS
        const u32 k = k_ring + x % 3 * TILE;
        w.wait(k_full + 8 * (x % 3), x / 3 & 1);
        if (pad_from(x) < ROWS) clear_rows<D>(k, pad_from(x));
        if (x >= GROUPS) w.wait(k_empty + 8 * ((x - GROUPS) % 3), (x - GROUPS) / 3 & 1);
        fence_after();
        if (elected() && !w.dead) {
          multiply_along_tmem<D>(tmem + x % GROUPS * ROWS, tmem_q, k, ins_s);
          commit(s_full + 8 * (x % GROUPS));
        }
        __syncwarp();
      };
      auto d_probabilities = [&](int x) {        // dP = dO V^T, over S, which has been read
        const int two = x & 1, at = x % GROUPS;
        const u32 v = v_ring + two * TILE;
        w.wait(v_full + 8 * two, x >> 1 & 1);
        if (pad_from(x) < ROWS) clear_rows<D>(v, pad_from(x));
        w.wait(s_read + 8 * at, x / GROUPS & 1);
        fence_after();
        if (elected() && !w.dead) {
          multiply_along_tmem<D>(tmem + at * ROWS, tmem_do, v, ins_dp);
          commit(dp_full + 8 * at);
          commit(v_empty + 8 * two);
        }
        __syncwarp();
      };
      w.wait(in_tmem, 0);
      fence_after();
      for (int x = 0; x < min(total, GROUPS); ++x) scores(x);
      for (int x = 0; x < total; x += GROUPS) {
#pragma unroll
        for (int y = x; y < x + GROUPS; ++y)
          if (y < total) d_probabilities(y);
#pragma unroll
        for (int y = x + GROUPS; y < x + 2 * GROUPS; ++y)
          if (y < total) scores(y);
      }
    }
  } else {
    give_registers<Block::left>();
  }
  linger(w.dead);
  wait_for_earlier();          // k_keys: this kernel ends behind it, as whatever follows in the stream expects
  fence_before();
  __syncthreads();
  if (warp == MMA_WARP) {
    fence_after();
    tmem_free(tmem, Block::columns);
  }
}

// The chunks' shares of dQ, or of dV and dK, added in their order: a warp a row.
template <class T, int D, bool KEYS>
__global__ void __launch_bounds__(256) k_join_gradients(const Args a) {
  wait_for_earlier();
  const int lane = threadIdx.x % 32, at = KEYS ? blockIdx.x / 2 : blockIdx.x, which = KEYS ? blockIdx.x % 2 : 0;
  const int r = at * 8 + threadIdx.x / 32, h = blockIdx.y, b = blockIdx.z, len = KEYS ? a.k_len : a.q_len;
  if (r >= len) return;
  const Lengths l = lengths_of(a, b);
  const int tile = r / ROWS * ROWS;
  int chunks;
  if (KEYS) chunks = r < l.m ? chunks_of(max(0, (l.n + ROWS - 1) / ROWS - first_query_tile(a, l, tile)) * ROWS) : 0;
  else chunks = end_of(a, l, r) > 0 ? chunks_of(key_tiles(a, l, tile) * ROWS) : 0;
  float sum[D / 32] = {};
  for (int s = 0; s < chunks; ++s) {
    const u64 slice = KEYS ? (u64)(2 * s + which) * a.batch + b : (u64)s * a.batch + b;
    const float* const from = a.parts + ((slice * (KEYS ? a.kv_heads : a.heads) + h) * len + r) * D;
#pragma unroll
    for (int e = 0; e < D / 32; ++e) sum[e] += from[lane + 32 * e];
  }
  T* const to = row_of<T>(KEYS ? (which ? a.d_k : a.d_v) : a.d_q, b, r, h);
#pragma unroll
  for (int e = 0; e < D / 32; ++e)
    if (lane + 32 * e < a.dim) to[lane + 32 * e] = narrow<T>(sum[e]);
}

// ------------------------------------------------------------------ host
typedef CUresult (*EncodeTiled)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                                const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
EncodeTiled encoder() {
  static const EncodeTiled f = [] {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult found;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &found) != cudaSuccess ||
        found != cudaDriverEntryPointSuccess)
      p = nullptr;
    return (EncodeTiled)p;
  }();
  return f;
}

// a tensor [batch][len][heads][dim] as tiles of 128 tokens and 64 elements
bool encode(CUtensorMap& map, u32 dtype, const ps_heads& h, int batch, int len, int heads, int dim) {
  const cuuint64_t extents[4] = {(cuuint64_t)dim, (cuuint64_t)heads, (cuuint64_t)len, (cuuint64_t)batch};
  const cuuint64_t strides[3] = {h.head_stride * 2, h.token_stride * 2, h.batch_stride * 2};
  const cuuint32_t box[4] = {64, 1, (cuuint32_t)ROWS, 1}, steps[4] = {1, 1, 1, 1};
  return encoder()(&map, dtype == PS_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 4, h.data, extents,
                   strides, box, steps, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                   CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

Args args_of(const AttentionArgs& a) {
  Args r;
  r.out = a.out; r.d_q = a.d_q; r.d_k = a.d_k; r.d_v = a.d_v;
  r.lse = a.lse; r.q_lens = a.q_lens; r.k_lens = a.k_lens;
  r.batch = a.batch; r.q_len = a.q_len; r.k_len = a.k_len; r.heads = a.heads; r.kv_heads = a.kv_heads; r.dim = a.dim;
  r.causal = a.causal;
  r.scale = a.scale;
  r.c = fmaxf(fabsf(a.scale) * LOG2E, 1e-30f);
  r.padded = (a.q_len + ROWS - 1) / ROWS * ROWS;
  const size_t rows = (size_t)a.batch * a.heads * r.padded;
  r.lse2 = (float*)a.work;
  r.delta = r.lse2 + rows;
  r.norms = (u32*)(r.delta + rows);
  r.rows_there = r.norms + 2 * (size_t)a.batch * a.kv_heads;
  r.parts = r.part_lse = nullptr;
  r.status = a.status;
  return r;
}

// Tensor memory is shared by the blocks of an SM, and each takes all of it: shared memory keeps a second block away.
u32 smem_for(int tiles, int d, u32 more) {
  const u32 want = tiles * PANEL * (d / 64) + more;
  return want < 120 * 1024 ? 120 * 1024 : want;
}
// (once a kernel and device: the call takes half a microsecond)
template <class K>
cudaError_t allow(K kernel, u32 smem, std::atomic<u64>& done) {
  int device = 0;
  cudaError_t e = cudaGetDevice(&device);
  if (e != cudaSuccess || (device < 64 && (done.load(std::memory_order_relaxed) >> device & 1))) return e;
  e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
  if (e == cudaSuccess && device < 64) done.fetch_or((u64)1 << device, std::memory_order_relaxed);
  return e;
}

template <class T, int D>
cudaError_t forward(u32 dtype, const AttentionArgs& a, cudaStream_t stream) {
  CUtensorMap q, k, v;
  if (!encode(q, dtype, a.q, a.batch, a.q_len, a.heads, a.dim)) return cudaErrorInvalidValue;
  if (a.k_len == 0) {
    k = v = q;                    // there are no keys: never read
  } else if (!encode(k, dtype, a.k, a.batch, a.k_len, a.kv_heads, a.dim) || !encode(v, dtype, a.v, a.batch, a.k_len, a.kv_heads, a.dim)) {
    return cudaErrorInvalidValue;
  }
  const u32 smem = smem_for(6, D, 1024), grid = (u32)((a.q_len + 2 * ROWS - 1) / (2 * ROWS)) * a.heads * a.batch;
  Args r = args_of(a);
  cudaError_t e;
  if (chunked(a.q_len, a.k_len)) {
    const int chunks = chunks_of(a.k_len);
    r.parts = (float*)a.work;
    r.part_lse = r.parts + (u64)chunks * a.batch * a.heads * a.q_len * D;
    static std::atomic<u64> allowed{0};
    if ((e = allow(k_forward<T, D, true>, smem, allowed)) != cudaSuccess) return e;
    k_forward<T, D, true><<<dim3(grid, chunks), THREADS, smem, stream>>>(q, k, v, r);
    if ((e = cudaGetLastError()) != cudaSuccess) return e;
    return launch_next(k_join_outputs<T, D>, dim3((a.q_len + 7) / 8, a.heads, a.batch), 256, 0, stream, r, chunks);
  }
  static std::atomic<u64> allowed{0};
  if ((e = allow(k_forward<T, D, false>, smem, allowed)) != cudaSuccess) return e;
  k_forward<T, D, false><<<grid, THREADS, smem, stream>>>(q, k, v, r);
  return cudaGetLastError();
}

// the backward pass's work buffer: both vectors of the padded rows, the norms and whether the rows are there, then the chunks' shares
size_t rows_bytes(const AttentionArgs& a) {
  const size_t padded = ((size_t)a.q_len + ROWS - 1) / ROWS * ROWS;
  return (sizeof(float) * 2 * a.batch * a.heads * padded + sizeof(u32) * (2 * (size_t)a.batch * a.kv_heads + 1) + 255) / 256 * 256;
}

template <class T, int D>
cudaError_t backward(u32 dtype, const AttentionArgs& a, cudaStream_t stream) {
  Args r = args_of(a);
  r.parts = (float*)((char*)a.work + rows_bytes(a));
  CUtensorMap q, k, v, d;
  if (a.q_len && (!encode(q, dtype, a.q, a.batch, a.q_len, a.heads, a.dim) || !encode(d, dtype, a.d_out, a.batch, a.q_len, a.heads, a.dim)))
    return cudaErrorInvalidValue;
  if (a.k_len && (!encode(k, dtype, a.k, a.batch, a.k_len, a.kv_heads, a.dim) || !encode(v, dtype, a.v, a.batch, a.k_len, a.kv_heads, a.dim)))
    return cudaErrorInvalidValue;
  if (!a.q_len) q = d = k;        // on one side there is nothing: never read
  if (!a.k_len) k = v = q;
  cudaError_t e;
  if constexpr (Range<T>::small) {
    e = cudaMemsetAsync(r.norms, 0, sizeof(u32) * 2 * a.batch * a.kv_heads, stream);
    if (e == cudaSuccess && a.k_len) {
      k_rows<T, D, false><<<dim3((a.k_len + ROWS_A_BLOCK<D> - 1) / ROWS_A_BLOCK<D>, a.kv_heads, a.batch), 256, 0, stream>>>(a.v, a.v, r);
      e = cudaGetLastError();
    }
    if (e != cudaSuccess) return e;
  }
  if (a.q_len) {
    k_rows<T, D, true><<<dim3((r.padded + ROWS_A_BLOCK<D> - 1) / ROWS_A_BLOCK<D>, a.heads, a.batch), 256, 0, stream>>>(a.d_out, a.out, r);
    if ((e = cudaGetLastError()) != cudaSuccess) return e;
  }
  // (one side at most is cut: few rows of it and many of the other)
  const bool cut_queries = chunked(a.k_len, a.q_len), cut_keys = chunked(a.q_len, a.k_len);
  if (a.k_len) {
    const u32 smem = smem_for(7, D, 5 * ROWS * 4 + sizeof(Shared)), grid = (u32)((a.k_len + ROWS - 1) / ROWS) * a.kv_heads * a.batch;
    static std::atomic<u64> allowed{0}, allowed_cut{0};
    if ((e = cut_queries ? allow(k_keys<T, D, true>, smem, allowed_cut) : allow(k_keys<T, D, false>, smem, allowed)) != cudaSuccess) return e;
    e = cut_queries ? launch_next(k_keys<T, D, true>, dim3(grid, chunks_of(a.q_len)), THREADS, smem, stream, q, k, v, d, r)
                    : launch_next(k_keys<T, D, false>, grid, THREADS, smem, stream, q, k, v, d, r);
    if (e != cudaSuccess) return e;
  }
  if (a.q_len) {
    const u32 smem = D == 64 ? 7 * PANEL + sizeof(Shared) : smem_for(7, D, sizeof(Shared)), threads = QueryBlock<D>::threads, grid = (u32)(r.padded / ROWS) * a.heads * a.batch;
    static std::atomic<u64> allowed{0}, allowed_cut{0};
    if ((e = cut_keys ? allow(k_queries<T, D, true>, smem, allowed_cut) : allow(k_queries<T, D, false>, smem, allowed)) != cudaSuccess) return e;
    if (cut_keys) {
      e = launch_next(k_queries<T, D, true>, dim3(grid, chunks_of(a.k_len)), threads, smem, stream, q, k, v, d, r);
    } else if (a.k_len) {
      e = launch_next(k_queries<T, D, false>, grid, threads, smem, stream, q, k, v, d, r);
    } else {
      k_queries<T, D, false><<<grid, threads, smem, stream>>>(q, k, v, d, r);      // (no kernel is between it and the rows)
      e = cudaGetLastError();
    }
    if (e != cudaSuccess) return e;
  }
  if (cut_keys) return launch_next(k_join_gradients<T, D, false>, dim3((a.q_len + 7) / 8, a.heads, a.batch), 256, 0, stream, r);
  if (cut_queries) return launch_next(k_join_gradients<T, D, true>, dim3((a.k_len + 7) / 8 * 2, a.kv_heads, a.batch), 256, 0, stream, r);
  return cudaSuccess;
}

}  // namespace

cudaError_t launch_attention_forward(u32 dtype, const AttentionArgs& a, int, cudaStream_t stream) {
  if (!encoder()) return cudaErrorNotSupported;
  if (dtype == PS_BF16) return a.dim <= 64 ? forward<__nv_bfloat16, 64>(dtype, a, stream) : forward<__nv_bfloat16, 128>(dtype, a, stream);
  return a.dim <= 64 ? forward<__half, 64>(dtype, a, stream) : forward<__half, 128>(dtype, a, stream);
}

size_t attention_forward_bytes(const AttentionArgs& a) {
  if (!chunked(a.q_len, a.k_len)) return 0;
  return sizeof(float) * chunks_of(a.k_len) * a.batch * a.heads * a.q_len * ((a.dim <= 64 ? 64 : 128) + 1);
}

size_t attention_backward_bytes(const AttentionArgs& a) {
  size_t parts = 0;
  if (chunked(a.q_len, a.k_len)) parts = (size_t)chunks_of(a.k_len) * a.batch * a.heads * a.q_len;
  if (chunked(a.k_len, a.q_len)) parts = (size_t)chunks_of(a.q_len) * 2 * a.batch * a.kv_heads * a.k_len;
  return rows_bytes(a) + sizeof(float) * parts * (a.dim <= 64 ? 64 : 128);
}

cudaError_t launch_attention_backward(u32 dtype, const AttentionArgs& a, int, cudaStream_t stream) {
  if (!encoder()) return cudaErrorNotSupported;
  if (dtype == PS_BF16) return a.dim <= 64 ? backward<__nv_bfloat16, 64>(dtype, a, stream) : backward<__nv_bfloat16, 128>(dtype, a, stream);
  return a.dim <= 64 ? backward<__half, 64>(dtype, a, stream) : backward<__half, 128>(dtype, a, stream);
}
