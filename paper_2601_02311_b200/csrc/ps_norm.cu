// Layer norm and its gradients.
//
//   y = (x - mean) rstd w + b
//   g = dY w;  xn = (x - mean) rstd;  dX = rstd (g - <g> - xn <g xn>) + residual;  dW = sum_r dY xn;  dB = sum_r dY
//
// with < > the mean over a row.  A row is read once and stays in registers: its mean first, then the sum of squared
// distances from it, so that a large mean costs no digits.  (Nor do the mean's own roundings where it is far larger than the distances: see
// SUMS_ROUND.)  Bytes bound both passes; dW and dB are summed in the
// registers of the threads that own the columns while the rows pass, so that the backward pass reads each matrix once.
//
// Which thread has which columns depends on the width alone: packs of 16 bytes where the width is a multiple of one (read element by
// element where a row does not begin at 16 bytes), elements next to one another where it is not.  So a row's bits do not
// depend on where it lies, nor on the other rows.
//
// Measured, one B200: 65536 x 8192 bfloat16 forward 410 us (5.2 TB/s, 0.8 of a copy's rate; issue slots 68 %), backward with a residual 749 us (5.7 TB/s);
// 12301 x 5003 floats backward 155 us (4.8 TB/s).  A row's loads are bulk copies into a ring, several rows ahead: with loads into registers one row ahead
// the backward pass took 1050 us.
#include <algorithm>
#include <atomic>
#include <type_traits>
#include "ps_columns.cuh"
#include "ps_tensor.cuh"

namespace {
using namespace train;

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int m = 16; m > 0; m /= 2) v += __shfl_xor_sync(0xffffffffu, v, m);
  return v;
}

// Sums over the R threads of a row, the same bits in all of them: within a warp, then over the warps' sums in a tree.  One barrier a
// call: the next one uses the other half of the slots.
template <int R, int COUNT>
struct RowSum {
  float* slots;         // [2][COUNT][R / 32]
  int turn;
  __device__ __forceinline__ explicit RowSum(float* s) : slots(s), turn(0) {}
  __device__ __forceinline__ void over(float (&v)[COUNT]) {
#pragma unroll
    for (int i = 0; i < COUNT; ++i) v[i] = warp_sum(v[i]);
    if (R == 32) return __syncwarp();
    constexpr int WARPS = R / 32;
    float* const mine = slots + turn * COUNT * WARPS;
    turn ^= 1;
    if (threadIdx.x % 32 == 0)
#pragma unroll
      for (int i = 0; i < COUNT; ++i) mine[i * WARPS + threadIdx.x / 32] = v[i];
    asm volatile("bar.sync 1, %0;" ::"n"(R) : "memory");
#pragma unroll
    for (int i = 0; i < COUNT; ++i) {
      v[i] = mine[i * WARPS + threadIdx.x % WARPS];
#pragma unroll
      for (int m = WARPS / 2; m > 0; m /= 2) v[i] += __shfl_xor_sync(0xffffffffu, v[i], m);
    }
  }
};

// ---- Rows that are shared by the blocks of a cluster, each with a range of the columns: their sums go through one another's shared memory.
constexpr u32 CLUSTER_MOST = 8;
// As RowSum, over the R threads of each of the cluster's blocks: every warp sends its sums to all blocks, and arrives at their barriers.  (With the block's sum
// taken first, and sent by one warp, 8000 x 16384 backward took 315 us instead of 289.)
template <int R, int COUNT>
struct ClusterSum {
  static constexpr u32 WARPS = R / 32, SLOTS = 2 * COUNT * CLUSTER_MOST * WARPS;
  u32 slots, bars, rank, size, uses;
  tensor::Waiter& waiter;
  __device__ __forceinline__ ClusterSum(const float* s, const u64* b, tensor::Waiter& w)
      : slots(tensor::smem_address(s)), bars(tensor::smem_address(b)), rank(tensor::cluster_rank()), size(tensor::cluster_size()), uses(0), waiter(w) {}
  __device__ __forceinline__ void over(float (&v)[COUNT]) {
    const u32 turn = uses & 1, parity = uses / 2 & 1, lane = threadIdx.x % 32, bar = bars + 8 * turn;
    ++uses;
#pragma unroll
    for (int i = 0; i < COUNT; ++i) v[i] = warp_sum(v[i]);
    const auto slot = [&](u32 i, u32 n) { return slots + 4 * ((turn * COUNT + i) * CLUSTER_MOST * WARPS + n); };
    if (lane < size) {
#pragma unroll
      for (int i = 0; i < COUNT; ++i)
        asm volatile("{\n\t.reg .b32 a;\n\tmapa.shared::cluster.u32 a, %0, %1;\n\tst.shared::cluster.f32 [a], %2;\n\t}"
                     ::"r"(slot(i, rank * WARPS + threadIdx.x / 32)), "r"(lane), "f"(v[i]) : "memory");
      asm volatile("{\n\t.reg .b32 a;\n\tmapa.shared::cluster.u32 a, %0, %1;\n\tmbarrier.arrive.release.cluster.shared::cluster.b64 _, [a];\n\t}"
                   ::"r"(bar), "r"(lane) : "memory");
    }
    __syncwarp();
    waiter.template wait<true>(bar, parity);
    __syncwarp();
#pragma unroll
    for (int i = 0; i < COUNT; ++i) {
      v[i] = 0.f;
      for (u32 n = lane; n < size * WARPS; n += 32) {
        float f;
        asm volatile("ld.shared.f32 %0, [%1];" : "=f"(f) : "r"(slot(i, n)) : "memory");
        v[i] += f;
      }
      v[i] = warp_sum(v[i]);
    }
  }
};

// Rows on their way: a ring of stages in shared memory, each with a row of every array that is read, brought by bulk copies that a warp of its
// own starts.  (Started by a thread of the row's they took twice as long in all: the others wait for it at their next barrier.)
// A copy begins and ends at multiples of 16 bytes: where a row does not, the rest of its first and last 16 bytes comes with it and is not used.
constexpr u32 RING_MOST = 8;              // stages at most
__host__ __device__ constexpr u32 slot_of(u64 cols, u32 width) { return (u32)((cols * width + 16 + 127) / 128 * 128); }
struct Ring {
  u32 base, bars, slot, stages, arrays;     // shared addresses; bytes of a row's place
  __device__ __forceinline__ u32 at(u32 stage, u32 array) const { return base + (stage * arrays + array) * slot; }
  __device__ __forceinline__ u32 full(u32 stage) const { return bars + 8 * stage; }
  __device__ __forceinline__ u32 empty(u32 stage) const { return bars + 8 * (RING_MOST + stage); }
  template <class T>
  __device__ __forceinline__ static u32 lead(const ps_matrix& m, u64 r) { return (u32)reinterpret_cast<uintptr_t>((const T*)m.data + r * m.stride) & 15u; }
  // all threads of the block; `warps` read the rows
  __device__ __forceinline__ void begin(unsigned char* rows, u64* bar_at, int warps) {
    base = (tensor::smem_address(rows) + 127u) & ~127u, bars = tensor::smem_address(bar_at);
    if (threadIdx.x == 0) {
      for (u32 s = 0; s < stages; ++s) tensor::barrier_init(full(s), 1), tensor::barrier_init(empty(s), warps);
      tensor::fence_barrier_init();
    }
    __syncthreads();
  }
  // one thread: rows first, first + step, ... of up to three matrices
  template <class T>
  __device__ __forceinline__ void bring(tensor::Waiter& waiter, const ps_matrix& m0, const ps_matrix& m1, const ps_matrix& m2, u64 first, u64 step, u64 rows, u32 cols) const {
    u32 stage = 0, parity = 1, filled = 0;
    const char* p0 = (const char*)((const T*)m0.data + first * m0.stride);
    const char* p1 = (const char*)((const T*)m1.data + first * m1.stride);
    const char* p2 = (const char*)((const T*)m2.data + first * m2.stride);
    const u64 by0 = step * m0.stride * sizeof(T), by1 = step * m1.stride * sizeof(T), by2 = step * m2.stride * sizeof(T);
    const u32 bytes = cols * (u32)sizeof(T) + 15u;
    const auto head = [](const char* p) { return (u32)reinterpret_cast<uintptr_t>(p) & 15u; };
    const auto whole = [&](const char* p) { return (head(p) + bytes) & ~15u; };
    for (u64 r = first; r < rows; r += step) {
      waiter.wait(empty(stage), parity);
      if (waiter.dead) break;
      tensor::barrier_expect(full(stage), whole(p0) + (arrays > 1 ? whole(p1) : 0) + (arrays > 2 ? whole(p2) : 0));
      tensor::load_bytes(at(stage, 0), p0 - head(p0), whole(p0), full(stage));
      if (arrays > 1) tensor::load_bytes(at(stage, 1), p1 - head(p1), whole(p1), full(stage));
      if (arrays > 2) tensor::load_bytes(at(stage, 2), p2 - head(p2), whole(p2), full(stage));
      p0 += by0, p1 += by1, p2 += by2;
      filled = min(filled + 1, stages);
      if (++stage == stages) stage = 0, parity ^= 1;
    }
    // leave no copy in flight, also where a wait has run out
    tensor::Waiter last(waiter.status);
    for (; filled > 0; --filled) {
      if (stage == 0) stage = stages, parity ^= 1;
      --stage;
      last.wait(full(stage), parity ^ 1);
    }
  }
  // a warp: it has read the stage
  __device__ __forceinline__ void leave(u32& stage, u32& parity) const {
    __syncwarp();
    if (threadIdx.x % 32 == 0) tensor::barrier_arrive(empty(stage));
    if (++stage == stages) stage = 0, parity ^= 1;
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
  __device__ __forceinline__ u64 both(int e) const { return Pack<T, E>::both(p.w, e, (const T*)nullptr); }        // (e even)
  // The words stay, the floats that they were widened to do not: without it the compiler keeps those from one walk to the next, in registers
  // that are not there.
  __device__ __forceinline__ void forget() {
    if (sizeof(T) == 2)
#pragma unroll
      for (int i = 0; i < Pack<T, E>::WORDS; ++i) asm volatile("" : "+r"(p.w[i]));
  }
  __device__ __forceinline__ void put_both(int e, u64 v) {
    const float lo = split(v).x, hi = split(v).y;
    if (sizeof(T) == 4) p.w[e] = __float_as_uint(lo), p.w[e + 1] = __float_as_uint(hi);
    else p.w[e / 2] = Pack<T, E>::two(lo, hi, (const T*)nullptr);
  }
  // `wide`: rows begin at multiples of 16 bytes.  Columns behind `cols` are zeros.
  // elements e .. e + G - 1 out of a row in shared memory, G = N or 2
  __device__ static __forceinline__ void read(u32 (&w)[(PACKED ? 16 : 2 * (int)sizeof(T)) / 4], u32 row, int e, u32 cols, bool wide) {
    constexpr int G = PACKED ? N : 2;
#pragma unroll
    for (int i = 0; i < (PACKED ? 16 : 2 * (int)sizeof(T)) / 4; ++i) w[i] = 0;
    if constexpr (PACKED)
      if (wide) {
        if (column(e) < cols)
          asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(row + column(e) * (u32)sizeof(T)));
        return;
      }
#pragma unroll
    for (int i = 0; i < G; ++i)
      if (column(e + i) < cols) {
        const u32 at = row + column(e + i) * (u32)sizeof(T);
        if constexpr (sizeof(T) == 4) {
          asm volatile("ld.shared.u32 %0, [%1];" : "=r"(w[i]) : "r"(at));
        } else {
          unsigned short v;
          asm volatile("ld.shared.u16 %0, [%1];" : "=h"(v) : "r"(at));
          w[i / 2] |= (u32)v << (16 * (i % 2));
        }
      }
  }
  __device__ __forceinline__ void take(u32 row, u32 cols, bool wide) {
    constexpr int G = PACKED ? N : 2, W = G * (int)sizeof(T) / 4;
#pragma unroll
    for (int e = 0; e < E; e += G) {
      u32 w[W];
      read(w, row, e, cols, wide);
#pragma unroll
      for (int i = 0; i < W; ++i) p.w[e * (int)sizeof(T) / 4 + i] = w[i];
    }
  }
  // as the row's elements from `first` on
  __device__ __forceinline__ void store_at(T* row, int first, u32 cols, bool wide) const {
    if (PACKED && wide) {
#pragma unroll
      for (int e = 0; e < E; e += N)
        if (column(first + e) < cols) {
          const u32* const w = p.w + e * (int)sizeof(T) / 4;
          *reinterpret_cast<uint4*>(row + column(first + e)) = make_uint4(w[0], w[1], w[2], w[3]);
        }
    } else {
#pragma unroll
      for (int e = 0; e < E; ++e)
        if (column(first + e) < cols) {
          if (sizeof(T) == 4) reinterpret_cast<u32*>(row)[column(first + e)] = p.w[e];
          else reinterpret_cast<unsigned short*>(row)[column(first + e)] = (unsigned short)(p.w[e / 2] >> (16 * (e % 2)));
        }
    }
  }
  __device__ __forceinline__ void store(T* row, u32 cols, bool wide) const { store_at(row, 0, cols, wide); }
};

// the G elements of weight or bias that belong to elements e .. e + G - 1 of a Piece
template <class T, int G>
struct Vector {
  u32 w[G * sizeof(T) < 4 ? 1 : G * (int)sizeof(T) / 4];
  template <int R, bool PACKED>
  __device__ __forceinline__ void load(const T* from, int e, u32 cols, bool wide, float without) {
    typedef Piece<T, R, 64, PACKED> P;
    if (from == nullptr) {
#pragma unroll
      for (int i = 0; i < (int)(sizeof(w) / 4); ++i) w[i] = sizeof(T) == 4 ? __float_as_uint(without) : Pack<T, G>::two(without, without, (const T*)nullptr);
    } else if (PACKED && wide) {
      const u32 c = P::column(e);
      uint4 v = make_uint4(0, 0, 0, 0);
      if (c < cols) v = *reinterpret_cast<const uint4*>(from + c);
      w[0] = v.x, w[1] = v.y, w[G * (int)sizeof(T) / 4 > 2 ? 2 : 0] = v.z, w[G * (int)sizeof(T) / 4 > 3 ? 3 : 0] = v.w;
    } else {
#pragma unroll
      for (int i = 0; i < G; ++i) {
        const u32 c = P::column(e + i), b = c < cols ? P::bits(from + c) : 0;
        if (sizeof(T) == 4) w[i] = b;
        else w[i / 2] = i % 2 ? w[i / 2] | b << 16 : b;
      }
    }
  }
  __device__ __forceinline__ u64 both(int i) const { return Pack<T, G>::both(w, i, (const T*)nullptr); }
  __device__ __forceinline__ void forget() {          // (as Piece's)
    if (sizeof(T) == 2)
#pragma unroll
      for (int i = 0; i < (int)(sizeof(w) / 4); ++i) asm volatile("" : "+r"(w[i]));
  }
};
__device__ __forceinline__ u64 twice(float v) { return pair(v, v); }
__device__ __forceinline__ float together(u64 v) { return split(v).x + split(v).y; }

// what stands n elements behind `p`; what is not there stays null (a block of a cluster asks whether there is a residual)
template <class T> __device__ __forceinline__ void* moved(void* p, u32 n) { return p ? (T*)p + n : nullptr; }
template <class T> __device__ __forceinline__ const void* moved(const void* p, u32 n) { return p ? (const T*)p + n : nullptr; }

struct Wide {           // which rows begin at multiples of 16 bytes
  bool x, y, d_y, residual, d_x, weight, bias;
};

// s / n to the last place: the product with 1 / n, and what that leaves of s
__device__ __forceinline__ float quotient(float s, float n, float share) {
  const float q = s * share;
  return fmaf(fmaf(-q, n, s), share, q);
}
// Where the distances are far smaller than the mean itself, a mean that is off by a few units of its last place shows in them; equal numbers would have distances at
// all.  The quotient does not do that, but rounded sums do.  Sums of 16-bit numbers of one size are exact while their digits and the columns' together are 24, in
// other kernels another walk over such a row (out of the L2) finds the mean of the distances, which is what the mean is off by.  (With it 65536 x 8192 of
// bfloat16 took 439 us instead of 380 although no row needed it, for want of registers.)  All threads of a row have the same two numbers.
template <class T> constexpr u32 LARGEST_SUM = sizeof(T) == 4 ? 1 : std::is_same<T, __half>::value ? 1 << 13 : 1 << 16;
template <class T, u32 COLUMNS> constexpr bool SUMS_ROUND = COLUMNS > LARGEST_SUM<T>;
__device__ __forceinline__ bool far_from_zero(float mean, float variance) { return mean * mean > 16.f * variance; }
// the mean square distance, out of that from a mean that is `off`
__device__ __forceinline__ float less_square(float variance, float off) {
  const float v = fmaf(-off, off, variance);
  return v < 0.f ? 0.f : v;                     // (NaN stays)
}
// sqrt's reciprocal, the fast function's (off by up to 2 units) improved by a Newton step
__device__ __forceinline__ float reciprocal_root(float v) {
  const float y = rsqrtf(v), half = 0.5f * v;
  return v > 0.f && v < INFINITY ? y * fmaf(-half * y, y, 1.5f) : y;
}

template <int R, int COUNT, bool SHARED>
__device__ __forceinline__ auto sum_of(float* slots, u64* bars, tensor::Waiter& waiter) {
  if constexpr (SHARED) return ClusterSum<R, COUNT>(slots, bars, waiter);
  else return RowSum<R, COUNT>(slots);
}
// all threads of the cluster: its barriers are there before, and its memory until after, all sums
__device__ __forceinline__ void begin_sums(u64* bars, u32 arrivals) {
  if (threadIdx.x == 0) {
    for (int i = 0; i < 2; ++i) tensor::barrier_init(tensor::smem_address(bars + i), arrivals);
    tensor::fence_barrier_init();
  }
  __syncthreads();
  tensor::cluster_sync();
}
__device__ __forceinline__ void end_sums() {
  __syncwarp();
  tensor::cluster_sync();
}

// Blocks of an SM at most, by the threads of a row and a thread's bytes of it: about 1024 threads, or 512 where they hold sums as well.
__host__ __device__ constexpr int forward_blocks(int r, int bytes) { return r == 32 ? 16 : r == 64 ? 12 : r == 128 ? 6 : r == 256 ? 3 : bytes <= 64 ? 2 : 1; }
__host__ __device__ constexpr int backward_blocks(int r) { return r == 32 ? 8 : r == 64 ? 5 : r == 128 ? 3 : r == 256 ? 2 : 1; }

// Elements of a thread whose weights stay in its registers as well.  Of more they are read again for each row.
template <class T, int E> constexpr bool HELD = E * sizeof(T) <= 32;

// A block has a row at a time, a thread E elements of it; a warp beside them brings the rows to come.
// (At 16 bits a walk over the elements is issue slots as much as it is bytes: floats are taken two at a time, which took 65536 x 8192 from 545 us to 441.)
template <class T, int R, int E, bool PACKED, bool SHARED>
__global__ void __launch_bounds__(R + 32, forward_blocks(R, E * sizeof(T))) k_norm(const NormArgs args, const Wide wide, Ring ring, float count, float share, u32 each) {
  extern __shared__ unsigned char rows[];
  __shared__ float slots[SHARED ? ClusterSum<R, 1>::SLOTS : 2 * R / 32];
  __shared__ u64 bars[2 * RING_MOST + 2];
  NormArgs a = args;
  u32 blocks = 1, begin = 0;                    // that share a row, and the columns' range
  if (SHARED) {
    blocks = tensor::cluster_size(), begin = tensor::cluster_rank() * each;
    a.cols = min((u64)each, args.cols - begin);
    for (ps_matrix* m : {&a.x, &a.y}) m->data = moved<T>(m->data, begin);
    a.weight = moved<T>(a.weight, begin), a.bias = moved<T>(a.bias, begin);
  }
  const u32 cols = (u32)a.cols;
  const u64 row = blockIdx.x / blocks, step = gridDim.x / blocks;
  ring.begin(rows, bars, R / 32);
  if (SHARED) begin_sums(bars + 2 * RING_MOST, blocks * (R / 32));
  tensor::Waiter waiter(a.status);
  if (threadIdx.x >= R) {
    if (threadIdx.x == R) ring.bring<T>(waiter, a.x, a.x, a.x, row, step, a.rows, cols);
    if (SHARED) end_sums();
    return;
  }
  auto sum = sum_of<R, 1, SHARED>(slots, bars + 2 * RING_MOST, waiter);
  typedef Piece<T, R, E, PACKED> P;
  constexpr int G = PACKED ? P::N : 2;          // elements that lie, or are read, together
  constexpr bool HOLD = HELD<T, E>;
  Vector<T, G> weights[HOLD ? E / G : 1], biases[HOLD ? E / G : 1];
  if (HOLD)
#pragma unroll
    for (int e = 0; e < E; e += G) {
      weights[e / G].template load<R, PACKED>((const T*)a.weight, e, cols, wide.weight, 1.f);
      biases[e / G].template load<R, PACKED>((const T*)a.bias, e, cols, wide.bias, 0.f);
    }
  u32 stage = 0, parity = 0;
  T* to = (T*)a.y.data + row * a.y.stride;
  for (u64 r = row; r < a.rows; r += step, to += step * a.y.stride) {
    P x;
    waiter.wait(ring.full(stage), parity);
    x.take(ring.at(stage, 0) + Ring::lead<T>(a.x, r), cols, wide.x);
    float s[1];
    u64 part[2] = {0, 0};
#pragma unroll
    for (int e = 0; e < E; e += 2) part[e / 2 % 2] = add2(part[e / 2 % 2], x.both(e));
    ring.leave(stage, parity);
    s[0] = together(add2(part[0], part[1]));
    sum.over(s);
    float mean = quotient(s[0], count, share);
    u64 less = twice(-mean);
    part[0] = part[1] = 0;
    x.forget();
#pragma unroll
    for (int e = 0; e < E; e += G) {
      u64 more = 0;
#pragma unroll
      for (int i = 0; i < G; i += 2) {
        u64 d = add2(x.both(e + i), less);
        if (!PACKED) d = pair(P::column(e) < cols ? split(d).x : 0.f, P::column(e + 1) < cols ? split(d).y : 0.f);
        more = fma2(d, d, more);
      }
      if (!PACKED || P::column(e) < cols) part[e / G % 2] = add2(part[e / G % 2], more);
    }
    s[0] = together(add2(part[0], part[1]));
    sum.over(s);
    float square = s[0] * share;
    if (SUMS_ROUND<T, (SHARED ? CLUSTER_MOST : 1) * R * E> && far_from_zero(mean, square)) {
      const T* const again = (const T*)a.x.data + r * a.x.stride;      // (not written before all threads have the sum)
      s[0] = 0.f;
#pragma unroll 1
      for (u32 c = threadIdx.x; c < cols; c += R) s[0] += widen(again[c]) - mean;
      sum.over(s);
      const float off = s[0] * share;
      mean += off, less = twice(-mean), square = less_square(square, off);
    }
    const float rstd = reciprocal_root(square + a.eps);
    const u64 by = twice(rstd);
    x.forget();
#pragma unroll
    for (int e = 0; e < E; e += G) {
      Vector<T, G> w, b;
      if (HOLD) {
        w = weights[HOLD ? e / G : 0], b = biases[HOLD ? e / G : 0];
        w.forget(), b.forget();
      } else {
        asm volatile("" ::: "memory");          // (not all weights at once: there are no registers for it)
        w.template load<R, PACKED>((const T*)a.weight, e, cols, wide.weight, 1.f);
        b.template load<R, PACKED>((const T*)a.bias, e, cols, wide.bias, 0.f);
      }
#pragma unroll
      for (int i = 0; i < G; i += 2) x.put_both(e + i, fma2(add2(x.both(e + i), less), mul2(by, w.both(i)), b.both(i)));
    }
    x.store(to, cols, wide.y);
    if (threadIdx.x == 0 && begin == 0) {
      if (a.mean) a.mean[r] = mean;
      if (a.rstd) a.rstd[r] = rstd;
    }
  }
  if (SHARED) end_sums();
}

// ---- Rows of up to 256 columns, in the backward pass 64: up to 32 lanes have a row, 8 elements each, and a warp as many rows as it has lanes for.  (107040 rows of 4 columns: 27 us, with a block
// for each 115.  100000 of 250: 58 and 95 us forward, but 214 and 159 backward.)
constexpr int NARROW = 256, NARROW_GRAD = 64, NARROW_E = 8, NARROW_BLOCKS = 4, NARROW_GRAD_BLOCKS = 2;
__device__ __forceinline__ float lanes_sum(float v, u32 lanes) {
  for (u32 m = lanes / 2; m > 0; m /= 2) v += __shfl_xor_sync(0xffffffffu, v, m);
  return v;
}
template <class T>
__global__ void __launch_bounds__(256, NARROW_BLOCKS) k_norm_narrow(const NormArgs a, u32 lanes, float count, float share) {
  const u32 lane = threadIdx.x % lanes, cols = (u32)a.cols, at_once = 256 / lanes;
  float w[NARROW_E], b[NARROW_E];
#pragma unroll
  for (int e = 0; e < NARROW_E; ++e) {
    const u32 c = e * lanes + lane;
    w[e] = a.weight && c < cols ? widen(((const T*)a.weight)[c]) : 1.f;
    b[e] = a.bias && c < cols ? widen(((const T*)a.bias)[c]) : 0.f;
  }
  // (all lanes of a warp go round as often: they meet in the sums)
  for (u64 first = (u64)blockIdx.x * at_once; first < a.rows; first += (u64)gridDim.x * at_once) {
    const u64 r = first + threadIdx.x / lanes;
    const bool there = r < a.rows;
    float v[NARROW_E], sum = 0.f;
#pragma unroll
    for (int e = 0; e < NARROW_E; ++e) {
      const u32 c = e * lanes + lane;
      v[e] = there && c < cols ? widen(((const T*)a.x.data)[r * a.x.stride + c]) : 0.f;
      sum += v[e];
    }
    float mean = quotient(lanes_sum(sum, lanes), count, share);
    sum = 0.f;
#pragma unroll
    for (int e = 0; e < NARROW_E; ++e) {
      v[e] = e * lanes + lane < cols ? v[e] - mean : 0.f;
      sum = fmaf(v[e], v[e], sum);
    }
    float square = lanes_sum(sum, lanes) * share;
    const bool far = SUMS_ROUND<T, NARROW> && far_from_zero(mean, square);
    if (__any_sync(0xffffffffu, far)) {           // (the lanes meet in the sum, which is for the rows that need it)
      sum = 0.f;
#pragma unroll
      for (int e = 0; e < NARROW_E; ++e) sum += v[e];
      const float off = lanes_sum(sum, lanes) * share, moved = far ? mean + off - mean : 0.f;
      square = far ? less_square(square, off) : square, mean += moved;
#pragma unroll
      for (int e = 0; e < NARROW_E; ++e) v[e] -= moved;
    }
    const float rstd = reciprocal_root(square + a.eps);
    if (!there) continue;
#pragma unroll
    for (int e = 0; e < NARROW_E; ++e) {
      const u32 c = e * lanes + lane;
      if (c < cols) ((T*)a.y.data)[r * a.y.stride + c] = narrow<T>(fmaf(v[e], rstd * w[e], b[e]));
    }
    if (lane == 0) {
      if (a.mean) a.mean[r] = mean;
      if (a.rstd) a.rstd[r] = rstd;
    }
  }
}
template <class T, bool GRADS>
__global__ void __launch_bounds__(256, NARROW_GRAD_BLOCKS) k_norm_grad_narrow(const NormArgs a, u32 lanes, float share) {
  __shared__ float sums[2][8][NARROW_GRAD];
  const u32 lane = threadIdx.x % lanes, cols = (u32)a.cols, at_once = 256 / lanes;
  float w[NARROW_E], of_w[NARROW_E], of_b[NARROW_E];
#pragma unroll
  for (int e = 0; e < NARROW_E; ++e) {
    const u32 c = e * lanes + lane;
    w[e] = a.weight && c < cols ? widen(((const T*)a.weight)[c]) : 1.f;
    of_w[e] = of_b[e] = 0.f;
  }
  for (u64 first = (u64)blockIdx.x * at_once; first < a.rows; first += (u64)gridDim.x * at_once) {
    const u64 r = first + threadIdx.x / lanes;
    const bool there = r < a.rows;
    const float mean = there ? a.mean[r] : 0.f, rstd = there ? a.rstd[r] : 0.f;
    float xn[NARROW_E], g[NARROW_E], along = 0.f, across = 0.f;
#pragma unroll
    for (int e = 0; e < NARROW_E; ++e) {
      const u32 c = e * lanes + lane;
      const bool here = there && c < cols;
      xn[e] = here ? (widen(((const T*)a.x.data)[r * a.x.stride + c]) - mean) * rstd : 0.f;
      g[e] = here ? widen(((const T*)a.d_y.data)[r * a.d_y.stride + c]) : 0.f;
      if (GRADS) {
        of_w[e] = fmaf(g[e], xn[e], of_w[e]);
        of_b[e] += g[e];
      }
      g[e] = __fmul_rn(g[e], w[e]);       // (never one instruction with the sum: the same bits with GRADS and without)
      along += g[e];
      across = fmaf(g[e], xn[e], across);
    }
    along = -lanes_sum(along, lanes) * share, across = -lanes_sum(across, lanes) * share;
    if (!there) continue;
#pragma unroll
    for (int e = 0; e < NARROW_E; ++e) {
      const u32 c = e * lanes + lane;
      if (c < cols) {
        const float v = g[e] + fmaf(xn[e], across, along);
        ((T*)a.d_x.data)[r * a.d_x.stride + c] =
            narrow<T>(a.residual.data ? fmaf(rstd, v, widen(((const T*)a.residual.data)[r * a.residual.stride + c])) : rstd * v);
      }
    }
  }
  if (GRADS) {                  // the rows of a warp, then the warps
#pragma unroll
    for (int e = 0; e < NARROW_E; ++e) {
      for (u32 m = lanes; m < 32; m *= 2) {
        of_w[e] += __shfl_xor_sync(0xffffffffu, of_w[e], m);
        of_b[e] += __shfl_xor_sync(0xffffffffu, of_b[e], m);
      }
      if (threadIdx.x % 32 < lanes) {
        sums[0][threadIdx.x / 32][e * lanes + lane] = of_w[e];
        sums[1][threadIdx.x / 32][e * lanes + lane] = of_b[e];
      }
    }
    __syncthreads();
    for (u32 c = threadIdx.x; c < 2 * cols; c += 256) {
      const u32 which = c >= cols;
      float all = 0.f;
      for (int i = 0; i < 8; ++i) all += sums[which][i][c - which * cols];
      a.parts[(u64)blockIdx.x * 2 * cols + c] = all;
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
    float mean = s[0] / (float)a.cols;
    s[0] = 0.f;
    for (u32 c = threadIdx.x; c < a.cols; c += LONG) {
      const float d = widen(x[c]) - mean;
      s[0] = fmaf(d, d, s[0]);
    }
    sum.over(s);
    float square = s[0] / (float)a.cols;
    if (far_from_zero(mean, square)) {
      s[0] = 0.f;
      for (u32 c = threadIdx.x; c < a.cols; c += LONG) s[0] += widen(x[c]) - mean;
      sum.over(s);
      const float off = s[0] / (float)a.cols;
      mean += off, square = less_square(square, off);
    }
    const float rstd = 1.f / sqrtf(square + a.eps);
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

// GRADS: the sums over this block's rows for dW and dB go to parts[block][2][cols]: they and what the second walk needs of
// the first are what the registers are for; the weights are in shared memory.
template <class T, int R, bool PACKED, bool GRADS, bool SHARED>
__global__ void __launch_bounds__(R + 32, backward_blocks(R)) k_norm_grad(const NormArgs args, const Wide wide, Ring ring, float share, u32 each) {
  constexpr int E = 16;
  extern __shared__ unsigned char rows[];
  __shared__ float slots[SHARED ? ClusterSum<R, 2>::SLOTS : 2 * 2 * R / 32];
  __shared__ u64 bars[2 * RING_MOST + 2];
  NormArgs a = args;
  u32 blocks = 1, begin = 0;                    // that share a row, and the columns' range
  if (SHARED) {
    blocks = tensor::cluster_size(), begin = tensor::cluster_rank() * each;
    a.cols = min((u64)each, args.cols - begin);
    for (ps_matrix* m : {&a.x, &a.d_y, &a.residual, &a.d_x}) m->data = moved<T>(m->data, begin);
    a.weight = moved<T>(a.weight, begin);
  }
  const u32 cols = (u32)a.cols;
  const u64 row = blockIdx.x / blocks, step = gridDim.x / blocks;
  ring.begin(rows, bars, R / 32);
  if (SHARED) begin_sums(bars + 2 * RING_MOST, blocks * (R / 32));
  tensor::Waiter waiter(a.status);
  if (threadIdx.x >= R) {
    if (threadIdx.x == R) ring.bring<T>(waiter, a.x, a.d_y, a.residual, row, step, a.rows, cols);
    if (SHARED) end_sums();
    return;
  }
  auto sum = sum_of<R, 2, SHARED>(slots, bars + 2 * RING_MOST, waiter);
  typedef Piece<T, R, E, PACKED> P;
  constexpr int G = PACKED ? P::N : 2, W = G * (int)sizeof(T) / 4;        // elements that are read together, and their words
  typedef Pack<T, G> Group;
  const u32 w_row = ring.at(ring.stages, 0);    // the weights stand behind the stages
  for (u32 c = threadIdx.x; c < cols; c += R) {
    if constexpr (sizeof(T) == 4)
      asm volatile("st.shared.u32 [%0], %1;" ::"r"(w_row + 4 * c), "r"(a.weight ? P::bits((const T*)a.weight + c) : 0x3f800000u) : "memory");
    else
      asm volatile("st.shared.u16 [%0], %1;" ::"r"(w_row + 2 * c), "h"((unsigned short)(a.weight ? P::bits((const T*)a.weight + c) : Pack<T, 2>::two(1.f, 1.f, (const T*)nullptr))) : "memory");
  }
  asm volatile("bar.sync 1, %0;" ::"n"(R) : "memory");
  u64 of_w[E / 2], of_b[E / 2];                 // two columns each
#pragma unroll
  for (int e = 0; e < E / 2; ++e) of_w[e] = of_b[e] = 0;
  u32 stage = 0, parity = 0;
  T* to = (T*)a.d_x.data + row * a.d_x.stride;
  float next_mean = 0.f, next_rstd = 0.f;
  if (row < a.rows) next_mean = a.mean[row], next_rstd = a.rstd[row];
  for (u64 r = row; r < a.rows; r += step, to += step * a.d_x.stride) {
    const u64 less = twice(-next_mean), by = twice(next_rstd);
    if (r + step < a.rows) next_mean = a.mean[r + step], next_rstd = a.rstd[r + step];
    const u32 x_row = ring.at(stage, 0) + Ring::lead<T>(a.x, r), d_row = ring.at(stage, 1) + Ring::lead<T>(a.d_y, r);
    const u32 more_row = ring.at(stage, 2) + Ring::lead<T>(a.residual, r);          // (of a residual)
    waiter.wait(ring.full(stage), parity);
    float s[2];
    u64 of_g = 0, of_gx = 0, kept_xn[E / 2], kept_g[E / 2];
#pragma unroll
    for (int e = 0; e < E; e += G) {
      u32 x[W], d[W];
      P::read(x, x_row, e, cols, wide.x);
      P::read(d, d_row, e, cols, wide.d_y);
      u32 w[W];
      P::read(w, w_row, e, cols, true);
#pragma unroll
      for (int i = 0; i < G; i += 2) {
        const u64 xn = mul2(add2(Group::both(x, i, (const T*)nullptr), less), by), dy = Group::both(d, i, (const T*)nullptr), g = mul2(dy, Group::both(w, i, (const T*)nullptr));
        if (GRADS) {
          of_w[(e + i) / 2] = fma2(dy, xn, of_w[(e + i) / 2]);
          of_b[(e + i) / 2] = add2(of_b[(e + i) / 2], dy);
        }
        of_g = add2(of_g, g);
        of_gx = fma2(g, xn, of_gx);             // (g is 0 behind the last column)
        kept_xn[(e + i) / 2] = xn, kept_g[(e + i) / 2] = g;
      }
    }
    s[0] = together(of_g);
    s[1] = together(of_gx);
    sum.over(s);
    const u64 along = twice(-s[0] * share), across = twice(-s[1] * share);
#pragma unroll
    for (int e = 0; e < E; e += G) {
      u32 more[W] = {};
      if (a.residual.data) P::read(more, more_row, e, cols, wide.residual);
      Piece<T, R, G, PACKED> out;
#pragma unroll
      for (int i = 0; i < G; i += 2) {
        const u64 v = add2(kept_g[(e + i) / 2], fma2(kept_xn[(e + i) / 2], across, along));
        out.put_both(i, a.residual.data ? fma2(by, v, Group::both(more, i, (const T*)nullptr)) : mul2(by, v));
      }
      out.store_at(to, e, cols, wide.d_x);
    }
    ring.leave(stage, parity);
  }
  if (GRADS) {
    float* const into = a.parts + row * 2 * args.cols + begin;
#pragma unroll
    for (int e = 0; e < E; ++e)
      if (P::column(e) < cols) {
        into[P::column(e)] = e % 2 ? split(of_w[e / 2]).y : split(of_w[e / 2]).x;
        into[args.cols + P::column(e)] = e % 2 ? split(of_b[e / 2]).y : split(of_b[e / 2]).x;
      }
  }
  if (SHARED) end_sums();
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
u32 blocks_for(u64 rows, int resident, int sm_count) { return (u32)std::min<u64>(rows, (u64)sm_count * resident); }

// Blocks of an SM, and the ring that each has: as many blocks as `most` and have `wanted` stages in the SM's shared memory, and all the stages that they
// have room for beside `more` rows.
constexpr u32 ROOM = 224 * 1024;
struct Layout {
  int resident;
  Ring ring;
  u32 smem;
};
Layout layout_of(int most, u32 wanted, u64 cols, u32 width, u32 arrays, u32 more) {
  Layout l = {};
  l.ring.slot = slot_of(cols, width);
  l.ring.arrays = arrays;
  const u32 stage = l.ring.slot * arrays;
  l.resident = most;
  const auto stages = [&] { return (ROOM / l.resident - 2048 - more * l.ring.slot) / stage; };       // (a row is at most 64 KB)
  while (l.resident > 1 && (ROOM / l.resident < 2048 + more * l.ring.slot || stages() < wanted)) --l.resident;
  l.ring.stages = std::max(1u, std::min(RING_MOST, stages()));
  l.smem = l.ring.stages * stage + more * l.ring.slot + 128;
  return l;
}
Layout forward_layout(int threads, int bytes, u64 cols, u32 width) { return layout_of(forward_blocks(threads, bytes), 2, cols, width, 1, 0); }
// (Blocks of clusters wait for one another: two on an SM rather than many stages.  1596 x 19021 floats with a residual: 181 us, with one 461.)
Layout backward_layout(int threads, u64 cols, u32 width, u32 arrays, bool shared) {
  return layout_of(backward_blocks(threads), shared ? 2 : 4, cols, width, arrays, 1);
}
// (asked for once a kernel and device)
template <auto KERNEL>
struct Prepared {
  static cudaError_t smem(u32 bytes) {
    static std::atomic<u64> devices{0};
    if (bytes <= 47 * 1024) return cudaSuccess;
    int device;
    cudaError_t e = cudaGetDevice(&device);
    if (e != cudaSuccess || (device < 64 && devices.load() >> device & 1)) return e;
    e = cudaFuncSetAttribute(KERNEL, cudaFuncAttributeMaxDynamicSharedMemorySize, 224 * 1024);
    if (e == cudaSuccess && device < 64) devices |= (u64)1 << device;
    return e;
  }
};

// How a row is shared: by one block, or where it has more than 8192 columns (32 KB of floats) by a cluster of 2, 4 or 8, with `each` columns (whole
// packs) in a block.  Clusters of 4 or 8 do not fill all SMs of a GPC: `clusters` of them run at a time.
struct Sharing {
  u32 blocks, each, clusters;
};
constexpr u32 A_BLOCKS_COLUMNS = 8192;
constexpr int SMS = 148;
Sharing sharing_of(u64 cols, u32 a_block) {
  if (cols <= a_block) return {1, (u32)cols, SMS};
  for (u32 blocks : {2, 4, 8})
    if (cols <= (u64)blocks * a_block) return {blocks, (u32)(((cols + blocks - 1) / blocks + 7) / 8 * 8), blocks == 2 ? 74u : blocks == 4 ? 32u : 16u};
  return {0, 0, 0};
}
template <class... Parameters, class... Arguments>
cudaError_t launch_cluster(void (*kernel)(Parameters...), u32 grid, u32 cluster, u32 threads, u32 smem, cudaStream_t stream, const Arguments&... arguments) {
  cudaLaunchAttribute together;
  together.id = cudaLaunchAttributeClusterDimension;
  together.val.clusterDim.x = cluster, together.val.clusterDim.y = together.val.clusterDim.z = 1;
  cudaLaunchConfig_t config = {};
  config.gridDim = dim3(grid);
  config.blockDim = dim3(threads);
  config.dynamicSmemBytes = smem;
  config.stream = stream;
  config.attrs = &together;
  config.numAttrs = cluster > 1 ? 1 : 0;
  return cudaLaunchKernelEx(&config, kernel, Parameters(arguments)...);
}

u32 narrow_lanes(u64 cols) {
  u32 lanes = 1;
  while (lanes * NARROW_E < cols) lanes *= 2;
  return lanes;
}

// Threads of a row, by the width: as few as hold it in 16 elements each, of rows of up to 64 KB in more of 512 threads.  (16384 columns of bfloat16:
// 8000 rows, 143 us by one block, 223 by two.)
template <class T, int R, bool PACKED, bool SHARED = false, int E = 16>
cudaError_t forward(const NormArgs& a, const Wide& wide, const Sharing& sharing, int sm_count, cudaStream_t stream) {
  constexpr auto kernel = k_norm<T, R, E, PACKED, SHARED>;
  const Layout l = forward_layout(R, E * sizeof(T), sharing.each, sizeof(T));
  const cudaError_t e = Prepared<kernel>::smem(l.smem);
  if (e != cudaSuccess) return e;
  const u64 groups = std::min<u64>(a.rows, (u64)(SHARED ? (int)sharing.clusters : sm_count) * l.resident);
  return launch_cluster(kernel, (u32)groups * sharing.blocks, sharing.blocks, R + 32, l.smem, stream, a, wide, l.ring, (float)a.cols, 1.f / (float)a.cols, sharing.each);
}
template <class T, bool PACKED>
cudaError_t forward(const NormArgs& a, const Wide& wide, int sm_count, cudaStream_t stream) {
  if (a.cols <= NARROW) {
    const u32 lanes = narrow_lanes(a.cols), at_once = 256 / lanes;
    k_norm_narrow<T><<<blocks_for((a.rows + at_once - 1) / at_once, NARROW_BLOCKS, sm_count), 256, 0, stream>>>(a, lanes, (float)a.cols, 1.f / (float)a.cols);
    return cudaGetLastError();
  }
  constexpr u32 MOST = 65536 / sizeof(T);
  const Sharing s = a.cols <= MOST ? Sharing{1, (u32)a.cols, SMS} : sharing_of(a.cols, A_BLOCKS_COLUMNS);
  if (s.blocks == 0) {
    k_norm_long<T><<<blocks_for(a.rows, 2, sm_count), LONG, 0, stream>>>(a);
    return cudaGetLastError();
  }
  if (s.blocks > 1) return forward<T, 512, PACKED, true>(a, wide, s, sm_count, stream);
  if (a.cols <= 32 * 16) return forward<T, 32, PACKED>(a, wide, s, sm_count, stream);
  if (a.cols <= 64 * 16) return forward<T, 64, PACKED>(a, wide, s, sm_count, stream);
  if (a.cols <= 128 * 16) return forward<T, 128, PACKED>(a, wide, s, sm_count, stream);
  if (a.cols <= 256 * 16) return forward<T, 256, PACKED>(a, wide, s, sm_count, stream);
  if (a.cols <= 512 * 16) return forward<T, 512, PACKED>(a, wide, s, sm_count, stream);
  if (a.cols <= 512 * 32) return forward<T, 512, PACKED, false, 32>(a, wide, s, sm_count, stream);
  if constexpr (sizeof(T) == 2) return forward<T, 512, PACKED, false, 64>(a, wide, s, sm_count, stream);
  return cudaErrorInvalidValue;          // (not reached: a row of floats is shared from there on)
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

// The backward pass's shape: threads of a row or a cluster's block, 16 elements each (0: the long kernels), and rows at a time, which are the parts of the
// sums; a block has four rows at least.  (A number for 148 SMs, whatever the device has: the sums' order depends on the sizes, and on whether there is a
// residual, alone.)
struct Shape {
  int threads;
  u32 groups;
  Sharing sharing;
};
constexpr int LANES = 1;                  // threads of narrow rows
Shape backward_shape(u32 width, u64 rows, u64 cols, u32 arrays) {
  if (cols <= NARROW_GRAD) {
    const u64 at_once = 256 / narrow_lanes(cols);
    return {LANES, (u32)std::max<u64>(1, std::min<u64>((rows + 2 * at_once - 1) / (2 * at_once), SMS * NARROW_GRAD_BLOCKS)), {}};
  }
  // two stages and the weights have to fit: of floats with more than 4096 columns not always
  const bool fits = cols <= A_BLOCKS_COLUMNS && (2 * arrays + 1) * slot_of(cols, width) <= ROOM - 2048;
  Shape s = {0, 0, sharing_of(cols, width == 2 || fits ? A_BLOCKS_COLUMNS : A_BLOCKS_COLUMNS / 2)};
  if (s.sharing.blocks == 0) {
    s.groups = (u32)std::max<u64>(1, std::min<u64>((rows + 63) / 64, 64));          // (chunks of rows)
    return s;
  }
  s.threads = s.sharing.blocks > 1 ? (width == 2 ? 512 : 256) : 32;
  while (s.threads < 512 && s.sharing.each > (u64)s.threads * 16) s.threads *= 2;
  s.groups = (u32)std::max<u64>(1, std::min<u64>((rows + 3) / 4, s.sharing.clusters * backward_layout(s.threads, s.sharing.each, width, arrays, s.sharing.blocks > 1).resident));
  return s;
}
template <class T, int R, bool PACKED, bool GRADS, bool SHARED>
cudaError_t backward(const NormArgs& a, const Wide& wide, const Shape& s, cudaStream_t stream) {
  constexpr auto kernel = k_norm_grad<T, R, PACKED, GRADS, SHARED>;
  const Layout l = backward_layout(R, s.sharing.each, sizeof(T), a.residual.data ? 3 : 2, SHARED);
  const cudaError_t e = Prepared<kernel>::smem(l.smem);
  if (e != cudaSuccess) return e;
  return launch_cluster(kernel, s.groups * s.sharing.blocks, s.sharing.blocks, R + 32, l.smem, stream, a, wide, l.ring, 1.f / (float)a.cols, s.sharing.each);
}
template <class T, int R, bool PACKED, bool SHARED = false>
cudaError_t backward(const NormArgs& a, const Wide& wide, const Shape& s, cudaStream_t stream) {
  return a.parts ? backward<T, R, PACKED, true, SHARED>(a, wide, s, stream) : backward<T, R, PACKED, false, SHARED>(a, wide, s, stream);
}
template <class T, bool PACKED>
cudaError_t backward(const NormArgs& a, const Shape& s, int sm_count, cudaStream_t stream) {
  const Wide wide = wide_of(a, sizeof(T));
  if (s.threads == LANES) {
    if (a.parts) k_norm_grad_narrow<T, true><<<s.groups, 256, 0, stream>>>(a, narrow_lanes(a.cols), 1.f / (float)a.cols);
    else k_norm_grad_narrow<T, false><<<s.groups, 256, 0, stream>>>(a, narrow_lanes(a.cols), 1.f / (float)a.cols);
    return cudaGetLastError();
  }
  if (s.sharing.blocks > 1) return backward<T, sizeof(T) == 2 ? 512 : 256, PACKED, true>(a, wide, s, stream);
  if (s.threads == 32) return backward<T, 32, PACKED>(a, wide, s, stream);
  if (s.threads == 64) return backward<T, 64, PACKED>(a, wide, s, stream);
  if (s.threads == 128) return backward<T, 128, PACKED>(a, wide, s, stream);
  if (s.threads == 256) return backward<T, 256, PACKED>(a, wide, s, stream);
  if (s.threads == 512) return backward<T, 512, PACKED>(a, wide, s, stream);
  if (a.parts) {                 // before d_x, which may stand in the place of d_y or x
    k_norm_columns<T><<<dim3((u32)((a.cols + 255) / 256), s.groups), 256, 0, stream>>>(a, (a.rows + s.groups - 1) / s.groups);
    const cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return e;
  }
  if (a.rows == 0) return cudaSuccess;
  k_norm_grad_long<T><<<blocks_for(a.rows, 2, sm_count), LONG, 0, stream>>>(a);
  return cudaGetLastError();
}
template <class T>
cudaError_t backward(const NormArgs& a, int sm_count, cudaStream_t stream) {
  const Shape s = backward_shape(sizeof(T), a.rows, a.cols, a.residual.data ? 3 : 2);
  if (a.rows == 0 && !a.parts) return cudaSuccess;
  const cudaError_t e = a.cols % (16 / sizeof(T)) == 0 ? backward<T, true>(a, s, sm_count, stream) : backward<T, false>(a, s, sm_count, stream);
  if (e != cudaSuccess || !a.parts) return e;
  return join_columns(a.grad_dtype, a.parts, s.groups, 2, a.cols, a.d_weight, a.d_bias, a.accumulate, stream);
}

}  // namespace

cudaError_t launch_norm_forward(u32 dtype, const NormArgs& a, int sm_count, cudaStream_t stream) {
  if (dtype == PS_F32) return forward<float>(a, sm_count, stream);
  return dtype == PS_BF16 ? forward<__nv_bfloat16>(a, sm_count, stream) : forward<__half>(a, sm_count, stream);
}

size_t norm_backward_bytes(u32 dtype, const NormArgs& a) {
  const u32 width = dtype == PS_F32 ? 4 : 2, groups = std::max(backward_shape(width, a.rows, a.cols, 2).groups, backward_shape(width, a.rows, a.cols, 3).groups);
  return (size_t)groups * 2 * a.cols * sizeof(float);
}

cudaError_t launch_norm_backward(u32 dtype, const NormArgs& a, int sm_count, cudaStream_t stream) {
  if (dtype == PS_F32) return backward<float>(a, sm_count, stream);
  return dtype == PS_BF16 ? backward<__nv_bfloat16>(a, sm_count, stream) : backward<__half>(a, sm_count, stream);
}
