// The fifth-generation tensor cores' instructions as the attention kernels use them: tiles of 16-bit
// elements in shared memory (128-byte swizzle, written by tiled bulk copies), accumulators in tensor
// memory, mbarriers between the roles of a block.
//
// A tile of R rows and 64 * n columns is n panels of [R][64] elements: a row of a panel is 128 bytes, its eight
// 16-byte pieces permuted by the row's number mod 8.  The same tile serves as an operand whose contraction runs along its rows
// (desc_along) and as one whose contraction runs across them (desc_across).
#pragma once
#include <cuda.h>
#include "ps_train.cuh"

namespace tensor {

constexpr int ROWS = 128;               // rows of every tile
constexpr u32 PANEL = ROWS * 128;       // bytes

__device__ __forceinline__ u32 smem_address(const void* p) { return (u32)__cvta_generic_to_shared(p); }

// ---- barriers.  Every wait has an end: after two seconds without progress it reports, and the thread waits
// for nothing any more (dead), starts no copy and no product, and leaves with the others.
constexpr u64 PATIENCE_NS = 2000000000ull;

__device__ __forceinline__ u64 now_ns() {
  u64 t;
  asm volatile("mov.u64 %0, %globaltimer;" : "=l"(t));
  return t;
}
__device__ __forceinline__ void barrier_init(u32 bar, u32 count) {
  asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void barrier_arrive(u32 bar) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void barrier_expect(u32 bar, u32 bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ bool barrier_passed(u32 bar, u32 parity) {
  u32 ok;
  asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}"
               : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
  return ok != 0;
}
struct Waiter {
  volatile u32* status;
  bool dead;
  __device__ __forceinline__ explicit Waiter(volatile u32* s) : status(s), dead(false) {}
  __device__ __forceinline__ void wait(u32 bar, u32 parity) {
    if (dead || barrier_passed(bar, parity)) return;
    const u64 begin = now_ns();
    while (!barrier_passed(bar, parity))
      if (now_ns() - begin > PATIENCE_NS) {
        dead = true;
        report(status, ST_TIMEOUT);
        return;
      }
  }
};

// ---- copies
__device__ __forceinline__ void fence_barrier_init() { asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory"); }
// writes of ordinary stores to shared memory, made visible to the tensor cores and the copy engine
__device__ __forceinline__ void fence_async() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

// 128 rows of one head, from row `row` on, into the panels of a tile; rows and columns that the tensor does not have read
// as zeros.  The map's dimensions: element, head, token, sequence.
template <int D>
__device__ __forceinline__ void load_tile(u32 to, const CUtensorMap* map, int head, int row, int batch, u32 bar) {
#pragma unroll
  for (int p = 0; p < D / 64; ++p)
    asm volatile(
        "cp.async.bulk.tensor.4d.shared::cta.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];"
        ::"r"(to + p * PANEL), "l"(map), "r"(p * 64), "r"(head), "r"(row), "r"(batch), "r"(bar) : "memory");
}
__device__ __forceinline__ void load_bytes(u32 to, const void* from, u32 bytes, u32 bar) {
  asm volatile("cp.async.bulk.shared::cta.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
               ::"r"(to), "l"(from), "r"(bytes), "r"(bar) : "memory");
}
// a warp: zeros in the rows of a tile from `first` on.  (All of its lanes, whether or not they still wait for anything: a wait may have run
// out for some of them alone, and the lanes meet at the end.)
template <int D>
__device__ __forceinline__ void clear_rows(u32 tile, int first) {
  for (int i = (int)(threadIdx.x % 32); i < (ROWS - first) * 8 * (D / 64); i += 32) {
    const int panel = i / ((ROWS - first) * 8), at = i - panel * (ROWS - first) * 8;
    asm volatile("st.shared.v4.u32 [%0], {%1, %1, %1, %1};" ::"r"(tile + panel * PANEL + first * 128 + at * 16), "r"(0) : "memory");
  }
  fence_async();
  __syncwarp();
}

// ---- tensor memory
__device__ __forceinline__ void tmem_alloc(u32 to_smem, u32 columns) {
  asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(to_smem), "r"(columns) : "memory");
  asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
}
__device__ __forceinline__ void tmem_free(u32 at, u32 columns) {
  asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(at), "r"(columns));
}
__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void wait_loads() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void wait_stores() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

#define PS_R8(v, o) "=r"(v[o]), "=r"(v[o + 1]), "=r"(v[o + 2]), "=r"(v[o + 3]), "=r"(v[o + 4]), "=r"(v[o + 5]), "=r"(v[o + 6]), "=r"(v[o + 7])
#define PS_I8(v, o) "r"(v[o]), "r"(v[o + 1]), "r"(v[o + 2]), "r"(v[o + 3]), "r"(v[o + 4]), "r"(v[o + 5]), "r"(v[o + 6]), "r"(v[o + 7])
// 32 columns of this thread's lane (its warp's quarter of the lanes is in the address)
__device__ __forceinline__ void tmem_load32(u32 (&v)[32], u32 at) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, "
      "%18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
      : PS_R8(v, 0), PS_R8(v, 8), PS_R8(v, 16), PS_R8(v, 24) : "r"(at));
}
__device__ __forceinline__ void tmem_load16(u32 (&v)[16], u32 at) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
      : PS_R8(v, 0), PS_R8(v, 8) : "r"(at));
}
__device__ __forceinline__ void tmem_store8(u32 at, const u32 (&v)[8]) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%8], {%0, %1, %2, %3, %4, %5, %6, %7};" ::PS_I8(v, 0), "r"(at) : "memory");
}
__device__ __forceinline__ void tmem_store32(u32 at, const u32 (&v)[32]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, "
      "%17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31};"
      ::PS_I8(v, 0), PS_I8(v, 8), PS_I8(v, 16), PS_I8(v, 24), "r"(at) : "memory");
}
__device__ __forceinline__ void tmem_store16(u32 at, const u32 (&v)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15};"
      ::PS_I8(v, 0), PS_I8(v, 8), "r"(at) : "memory");
}

// a tile's rows from shared memory to the lanes of tensor memory, by four warps: a thread has a row
template <int D>
__device__ __forceinline__ void tile_to_tmem(u32 at, u32 tile) {
  const u32 row = threadIdx.x % ROWS;
#pragma unroll
  for (int p = 0; p < D / 64; ++p) {
    u32 v[32];
#pragma unroll
    for (int c = 0; c < 8; ++c)
      asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];"
                   : "=r"(v[4 * c]), "=r"(v[4 * c + 1]), "=r"(v[4 * c + 2]), "=r"(v[4 * c + 3])
                   : "r"(tile + p * PANEL + row * 128 + ((c ^ (row & 7)) << 4)));
    tmem_store32(at + 32 * p, v);
  }
  wait_stores();
  fence_before();
  __syncwarp();
}

// ---- products
// Operand descriptors: start, leading and stride offsets in 16-byte units, 128-byte swizzle.  Of a tile's descriptors only the
// start differs, in the low word; a step of 16 along the contraction adds a constant to it.
constexpr u32 DESC_HIGH = 64u | (1u << 14) | (2u << 29);
__device__ __forceinline__ u32 desc_along(u32 tile) { return ((tile & 0x3FFFFu) >> 4) | (1u << 16); }         // contraction along the tile's columns
__device__ __forceinline__ u32 desc_across(u32 tile) { return ((tile & 0x3FFFFu) >> 4) | ((PANEL >> 4) << 16); }   // along its rows
__device__ __forceinline__ constexpr u32 step_along(int s) { return (s / 4) * (PANEL >> 4) + (s % 4) * 2; }
__device__ __forceinline__ constexpr u32 step_across(int s) { return s * 128; }

template <class T> struct Format;
template <> struct Format<__half> { static constexpr u32 code = 0; };
template <> struct Format<__nv_bfloat16> { static constexpr u32 code = 1; };
// 128 x n products with 32-bit sums; `across`: B's contraction runs along its tile's rows; `minus`: A is negated
template <class T>
__device__ __forceinline__ constexpr u32 instruction(int n, bool across, bool minus) {
  return (1u << 4) | (Format<T>::code << 7) | (Format<T>::code << 10) | ((minus ? 1u : 0u) << 13) | ((across ? 1u : 0u) << 16) |
         ((u32)(n >> 3) << 17) | ((u32)(128 >> 4) << 24);
}
// One lane of the warp, always the same one.  (With this instead of a comparison of the lane's number, and descriptors that advance by
// constants, 8192 queries with 32 heads of 128 took 472 us forward instead of 505, and 1595 backward instead of 1740.)
__device__ __forceinline__ bool elected() {
  u32 one;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(one));
  return one != 0;
}
__device__ __forceinline__ void mma_smem(u32 d, u32 a, u32 b, u32 ins, bool add) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t.reg .b64 a, b;\n\tsetp.ne.u32 p, %5, 0;\n\tmov.b64 a, {%1, %4};\n\tmov.b64 b, {%2, %4};\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %3, p;\n\t}"
      ::"r"(d), "r"(a), "r"(b), "r"(ins), "r"(DESC_HIGH), "r"(add ? 1u : 0u) : "memory");
}
__device__ __forceinline__ void mma_tmem(u32 d, u32 a, u32 b, u32 ins, bool add) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t.reg .b64 b;\n\tsetp.ne.u32 p, %5, 0;\n\tmov.b64 b, {%2, %4};\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], b, %3, p;\n\t}"
      ::"r"(d), "r"(a), "r"(b), "r"(ins), "r"(DESC_HIGH), "r"(add ? 1u : 0u) : "memory");
}
// d = a b^T: both tiles' contraction along their columns, D of them
template <int D>
__device__ __forceinline__ void multiply_along(u32 d, u32 a, u32 b, u32 ins) {
  const u32 x = desc_along(a), y = desc_along(b);
#pragma unroll
  for (int s = 0; s < D / 16; ++s) mma_smem(d, x + step_along(s), y + step_along(s), ins, s > 0);
}
// the same with a in tensor memory, D columns of 16 bits: only b's tile is read from shared memory, whose 128 bytes a cycle both
// tiles of 128 rows just use up
template <int D>
__device__ __forceinline__ void multiply_along_tmem(u32 d, u32 a, u32 b, u32 ins) {
  const u32 y = desc_along(b);
#pragma unroll
  for (int s = 0; s < D / 16; ++s) mma_tmem(d, a + 8 * s, y + step_along(s), ins, s > 0);
}
// d (+)= a b: a in tensor memory, its K columns of 16 bits against K rows of tile b
template <int K = ROWS>
__device__ __forceinline__ void multiply_across(u32 d, u32 a, u32 b, u32 ins, bool add) {
  const u32 y = desc_across(b);
#pragma unroll
  for (int s = 0; s < K / 16; ++s) mma_tmem(d, a + 8 * s, y + step_across(s), ins, add || s > 0);
}
// the barrier is arrived at once all products that this thread has issued are done
__device__ __forceinline__ void commit(u32 bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}

// ---- registers: a group of four warps gives some of its own up, another takes them
template <int N> __device__ __forceinline__ void give_registers() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N)); }
template <int N> __device__ __forceinline__ void take_registers() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N)); }

// ---- arithmetic, two floats an instruction where there is one
__device__ __forceinline__ u64 pair(float x, float y) {
  u64 r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(x), "f"(y));
  return r;
}
__device__ __forceinline__ float2 split(u64 v) {
  float2 r;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(v));
  return r;
}
__device__ __forceinline__ u64 fma2(u64 a, u64 b, u64 c) {
  u64 r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ u64 add2(u64 a, u64 b) {
  u64 r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ u64 mul2(u64 a, u64 b) {
  u64 r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// 2^(x c + y) of two numbers.  (The special-function pipe gives 16 results a cycle and SM.  A polynomial of degree 5 on the
// multiply-add pipe for every fourth pair made no kernel here faster by more than 3 %, and those with 128 columns slower.)
__device__ __forceinline__ float2 exp2_pair(u32 x0, u32 x1, u64 c, u64 y) {
  const float2 v = split(fma2(pair(__uint_as_float(x0), __uint_as_float(x1)), c, y));
  return make_float2(exp2_fast(v.x), exp2_fast(v.y));
}
template <class T> __device__ __forceinline__ u32 pack(float lo, float hi);
template <> __device__ __forceinline__ u32 pack<__nv_bfloat16>(float lo, float hi) {
  u32 r;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
template <> __device__ __forceinline__ u32 pack<__half>(float lo, float hi) {
  u32 r;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}

}  // namespace tensor
