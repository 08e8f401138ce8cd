// The linear layer with what follows it, and its gradients: matrix products on the fifth-generation tensor cores.
//
//   y = act(x W^T + bias) + residual                       C[t][o], sum over the inputs:  both matrices lie along the sum
//   dX = (dPre W) o act_below'(below) + residual           C[t][i], sum over the outputs: W lies across it
//   dW = dPre^T x                                          C[o][i], sum over the tokens:  both lie across it
//   dPre = dY o act'(pre),  dBias = sum_t dPre             elementwise and by columns, before the products
//
// One kernel does the three products.  A block (or a pair of blocks on two SMs, which share a tile of 256 x 256: each has
// half of both operands, and reads half as much from the L2 as alone) walks over tiles of C; a warp copies operands
// into a ring of shared memory, 64 columns of the sum at a time, a thread starts the products, whose sums stand in tensor memory twice
// over, and eight warps bring a finished tile to memory while the next one is being summed: add the bias, activate, multiply, add, round.
//
// The sum over the inputs (outputs) is never cut, and goes in the same order in tiles of any size, so a row of y or dX does not
// depend on what else the call computes.  The sum over the tokens is cut where dW has few tiles; a second kernel adds the parts in order.
//
// Measured, one B200: 16384 tokens, 8192 to 32768 columns with gelu, 5.7 ms in a burst (1.56 PFLOP/s; the library's plain product 5.4 to 5.6), 6.9 in a loop
// at the power limit; the tensor pipe is busy for 89 % of the time.  Its like's gradients 13.5 to 14 ms in a loop.  2048 x 4096 x 4096: 51 us (library 48).
#include <algorithm>
#include <atomic>
#include <type_traits>
#include "ps_columns.cuh"
#include "ps_tensor.cuh"

namespace {
using namespace train;
using namespace tensor;

constexpr int STEP = 64;                  // of the sum, a stage of the ring
constexpr int WRITERS = 8, COPY_WARP = 8, MMA_WARP = 9, TILE_WARP = 10, THREADS = 352;
constexpr u32 TILES_AHEAD = 2;            // answers that some roles have read and others not
// The next tile is asked for this many steps before the copies of one end: early enough for the ring to stay full, and no earlier, since a tile that is
// taken is lost to the blocks that have nothing to do
constexpr u32 ASK_BEFORE = 2;
constexpr int LOW_SHIFT = 12;             // see multiply_scaled
// Steps that a sum which leaves in 32 bits takes in tensor memory at a time; it is then added to what is there.  (The tensor cores cut off rather than round: each of the 16
// products of an instruction at a quarter of a unit of the sum's last place, the sum at a unit.  It draws a sum towards zero; rounded to 16 bits nobody sees it.  Error of
// the gradient, terms of both signs in bfloat16, with 64 steps at a time 4.4e-6, with 32 2.1e-6, with 24 1.5e-6, with 16 1.0e-6; 8192 tokens, 4096 to 4096
// columns, took 394 us with 64, 406 with 32 and 465 with 16.  Sums in plain floats are off by 1.0e-6.  Terms of one sign alone lose more, 3.1e-6 and, since half's
// products are longer, 8.2e-6; plain floats 1.4e-6.)
constexpr u32 STEPS_AT_ONCE = 24;
constexpr u32 BUFFER = 32 * 128;          // a warp's 32 rows of 128 bytes on their way from or to memory
constexpr u32 LEADER = 0xFEFFFFFFu;       // a shared-memory address, in the pair's first block

// What is computed: which product (WEIGHT_GRAD_TWO: of dPre in two parts), the type of its result, the tile's columns, and whether two
// blocks share it
enum Kind { OUTPUT, INPUT_GRAD, WEIGHT_GRAD, WEIGHT_GRAD_TWO };
template <class T_, class O_, Kind KIND_, int COLUMNS_, bool PAIR_>
struct Form {
  typedef T_ T;
  typedef O_ O;
  static constexpr Kind KIND = KIND_;
  static constexpr int COLUMNS = COLUMNS_;
  static constexpr bool PAIR = PAIR_;
  static constexpr bool TWO = KIND == WEIGHT_GRAD_TWO;
  static constexpr bool A_ACROSS = KIND == WEIGHT_GRAD || TWO, B_ACROSS = KIND != OUTPUT;
  static constexpr int B_ROWS = PAIR ? COLUMNS / 2 : COLUMNS;             // of this block
  static constexpr int B_LOADED = B_ACROSS ? (B_ROWS + 63) / 64 * 64 : B_ROWS;      // (panels of 64 come whole)
  static constexpr u32 A_BYTES = ROWS * STEP * 2, B_BYTES = B_LOADED * STEP * 2, STAGE = A_BYTES + B_BYTES;
  static constexpr u32 BUFFERS = WRITERS * 2 * BUFFER, AROUND = BUFFERS + WRITERS * 128 + 1024 + 320;   // (alignment, barriers, tiles)
  static constexpr int STAGES = (int)((227 * 1024 - AROUND) / STAGE) < 8 ? (int)((227 * 1024 - AROUND) / STAGE) : 8;
  static constexpr u32 SMEM = AROUND + STAGES * STAGE;
  static constexpr u32 SUM = COLUMNS <= 64 ? 64 : COLUMNS <= 128 ? 128 : 256, TMEM = 2 * SUM;      // columns of tensor memory
  static constexpr int CHUNK = 128 / sizeof(O);                           // columns of a buffer
  static_assert(STAGES >= 3 && COLUMNS % CHUNK == 0 && TMEM <= 512 && SMEM > 116 * 1024, "");   // (one block an SM: it takes tensor memory alone)
};

struct Product {
  u32 m, n, steps;                        // C's sizes, and stages of the sum
  u32 m_tiles, n_tiles, tiles, splits, steps_each, steps_at_once, stage_bytes;
  const void* bias;
  u32 activation, below_activation;
  u32 has_residual, has_below, has_pre, after;      // after: its tiles come behind the other product's
  ps_matrix out, pre;                     // the results, for what stores of boxes cannot write (see store_edge); out.data null: they can
  volatile u32* status;
};

// ---- activations and their derivatives, in 32 bits.  (Exponentials with the fast function's error, 2 + 1.2 |argument| units of 2^-23 relative to the value, quotients
// with one such unit: results in 16 bits hide it; gradients of weight and bias in 32 bits hold it.)
__device__ __forceinline__ float reciprocal(float v) {
  float r;                                          // (one unit off at most; 0 of infinity)
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
  return r;
}
__device__ __forceinline__ float sigmoid(float v) { return reciprocal(1.f + __expf(-v)); }
constexpr float LOG2_E = 1.44269504f, TANH_FACTOR = 0.79788456f, TANH_CUBE = 0.044715f;
// Phi(v), and e^(-v^2 / 2) on the way.  Phi(-|v|) = e^(-v^2 / 2) P(t), t = 1 / (1 + 0.34 |v|): P is a polynomial fitted to the quotient itself (least squares over
// 0 <= |v| <= 14, reweighted until the largest error stood still, with up to 11 times the relative error where the value is small).  In floats it is off by
// 1.8e-7 beside 1, and by 1.2e-6 of the value on the far side: a formula whose error is small beside 1 alone loses its digits there (one of 1.5e-7 had
// gelu(-6) wrong by 0.4 %).  Every instruction counts: 2048 tokens, 1024 to 4096 columns, take 24.9 us, and 26.8 with __expf in place
// of the instruction.
__device__ __forceinline__ float normal_share(float v, float& e) {
  const float t = reciprocal(fmaf(fabsf(v), 0.34f, 1.f));
  e = exp2_fast(v * v * (-0.5f * LOG2_E));
  const float near = fmaf(t, fmaf(t, fmaf(t, 0.0475229584f, -0.212724924f), 0.287034124f), -0.0539200082f);
  const float tail = fmaf(t, fmaf(t, fmaf(t, fmaf(t, near, 0.170085922f), 0.125248134f), 0.136808395f), -5.46155788e-05f) * e;
  return v >= 0.f ? 1.f - tail : tail;
}
template <int ACT>
__device__ __forceinline__ float activated(float v) {
  if (ACT == PS_ACT_RELU) return v > 0.f ? v : v != v ? v : 0.f;
  if (ACT == PS_ACT_GELU) {
    float e;
    return v * normal_share(v, e);
  }
  if (ACT == PS_ACT_GELU_TANH) return v * sigmoid(2.f * TANH_FACTOR * fmaf(TANH_CUBE * v * v, v, v));
  if (ACT == PS_ACT_SILU) return v * sigmoid(v);
  return v;
}
template <int ACT>
__device__ __forceinline__ float slope(float v) {
  if (ACT == PS_ACT_RELU) return v > 0.f ? 1.f : 0.f;
  if (ACT == PS_ACT_GELU) {
    float e;
    const float share = normal_share(v, e);
    return fmaf(v * (0.5f * TANH_FACTOR), e, share);
  }
  if (ACT == PS_ACT_GELU_TANH) {
    const float s = sigmoid(2.f * TANH_FACTOR * fmaf(TANH_CUBE * v * v, v, v));
    if (s * (1.f - s) == 0.f) return s;                     // (far out, where the other factor may be infinite)
    return fmaf(v * s * (1.f - s), 2.f * TANH_FACTOR * fmaf(3.f * TANH_CUBE * v, v, 1.f), s);
  }
  if (ACT == PS_ACT_SILU) {
    const float s = sigmoid(v);
    return s * fmaf(v, 1.f - s, 1.f);
  }
  return 1.f;
}
template <int N>
__device__ __forceinline__ void activate(u32 activation, float (&v)[N]) {
#define PS_EACH(ACT)   \
  if (activation == ACT) { _Pragma("unroll") for (int e = 0; e < N; ++e) v[e] = activated<ACT>(v[e]); }
  PS_EACH(PS_ACT_RELU) PS_EACH(PS_ACT_GELU) PS_EACH(PS_ACT_GELU_TANH) PS_EACH(PS_ACT_SILU)
#undef PS_EACH
}
template <int N>
__device__ __forceinline__ void times_slope(u32 activation, float (&v)[N], const float (&at)[N]) {
#define PS_EACH(ACT)   \
  if (activation == ACT) { _Pragma("unroll") for (int e = 0; e < N; ++e) v[e] *= slope<ACT>(at[e]); }
  PS_EACH(PS_ACT_RELU) PS_EACH(PS_ACT_GELU) PS_EACH(PS_ACT_GELU_TANH) PS_EACH(PS_ACT_SILU)
#undef PS_EACH
}

// ---- a pair's instructions
__device__ __forceinline__ void arrive_at_leader(u32 bar) {
  asm volatile("{\n\t.reg .b32 a;\n\tmapa.shared::cluster.u32 a, %0, 0;\n\tmbarrier.arrive.release.cluster.shared::cluster.b64 _, [a];\n\t}" ::"r"(bar) : "memory");
}
// A product whose sum goes on from what is there times 2^-LOW_SHIFT: so a matrix in two parts, the low one held 2^LOW_SHIFT times as large (16-bit floats
// of IEEE have no small numbers), needs one sum.
template <bool PAIR>
__device__ __forceinline__ void multiply_scaled(u32 d, u32 a, u32 b, u32 ins) {
  if (PAIR)
    asm volatile(
        "{\n\t.reg .pred p;\n\t.reg .b64 a, b;\n\tsetp.eq.u32 p, 0, 0;\n\tmov.b64 a, {%1, %4};\n\tmov.b64 b, {%2, %4};\n\t"
        "tcgen05.mma.cta_group::2.kind::f16 [%0], a, b, %3, p, %5;\n\t}"
        ::"r"(d), "r"(a), "r"(b), "r"(ins), "r"(DESC_HIGH), "n"(LOW_SHIFT) : "memory");
  else
    asm volatile(
        "{\n\t.reg .pred p;\n\t.reg .b64 a, b;\n\tsetp.eq.u32 p, 0, 0;\n\tmov.b64 a, {%1, %4};\n\tmov.b64 b, {%2, %4};\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %3, p, %5;\n\t}"
        ::"r"(d), "r"(a), "r"(b), "r"(ins), "r"(DESC_HIGH), "n"(LOW_SHIFT) : "memory");
}

// ---- copies of a box of two or three dimensions
template <bool PAIR>
__device__ __forceinline__ void load_box(u32 to, const CUtensorMap* map, int column, int row, u32 bar) {
  if (PAIR)
    asm volatile("cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
                 ::"r"(to), "l"(map), "r"(column), "r"(row), "r"(bar & LEADER) : "memory");
  else
    asm volatile("cp.async.bulk.tensor.2d.shared::cta.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
                 ::"r"(to), "l"(map), "r"(column), "r"(row), "r"(bar) : "memory");
}
__device__ __forceinline__ void load_rows(u32 to, const CUtensorMap* map, int column, int row, int part, u32 bar) {
  asm volatile("cp.async.bulk.tensor.3d.shared::cta.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
               ::"r"(to), "l"(map), "r"(column), "r"(row), "r"(part), "r"(bar) : "memory");
}
__device__ __forceinline__ void store_rows(const CUtensorMap* map, int column, int row, int part, u32 from) {
  asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.bulk_group [%0, {%1, %2, %3}], [%4];"
               ::"l"(map), "r"(column), "r"(row), "r"(part), "r"(from) : "memory");
}
__device__ __forceinline__ void commit_stores() { asm volatile("cp.async.bulk.commit_group;" ::: "memory"); }
__device__ __forceinline__ void wait_stores_read() { asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory"); }
__device__ __forceinline__ void wait_stores_done() { asm volatile("cp.async.bulk.wait_group 0;" ::: "memory"); }

// ---- products
constexpr u32 ACROSS_PANEL = STEP * 128;          // bytes of 64 columns by 64 steps of a sum across them
template <bool ACROSS>
__device__ __forceinline__ u32 descriptor(u32 tile) {
  return ((tile & 0x3FFFFu) >> 4) | (ACROSS ? (ACROSS_PANEL >> 4) << 16 : 1u << 16);
}
template <bool ACROSS>
__device__ __forceinline__ constexpr u32 step_of(int s) { return ACROSS ? s * 128 : s * 2; }
template <class F>
__device__ __forceinline__ constexpr u32 instruction_of() {
  return (1u << 4) | (Format<typename F::T>::code << 7) | (Format<typename F::T>::code << 10) | ((F::A_ACROSS ? 1u : 0u) << 15) |
         ((F::B_ACROSS ? 1u : 0u) << 16) | ((u32)(F::COLUMNS >> 3) << 17) | ((u32)((F::PAIR ? 256 : 128) >> 4) << 24);
}
template <bool PAIR>
__device__ __forceinline__ void multiply(u32 d, u32 a, u32 b, u32 ins, bool add) {
  if (PAIR)
    asm volatile(
        "{\n\t.reg .pred p;\n\t.reg .b64 a, b;\n\tsetp.ne.u32 p, %5, 0;\n\tmov.b64 a, {%1, %4};\n\tmov.b64 b, {%2, %4};\n\t"
        "tcgen05.mma.cta_group::2.kind::f16 [%0], a, b, %3, p;\n\t}"
        ::"r"(d), "r"(a), "r"(b), "r"(ins), "r"(DESC_HIGH), "r"(add ? 1u : 0u) : "memory");
  else
    mma_smem(d, a, b, ins, add);
}
// the barrier (of both blocks of a pair) is arrived at once the products started so far are done
template <bool PAIR>
__device__ __forceinline__ void commit_to(u32 bar) {
  if (PAIR)
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar), "h"((unsigned short)3) : "memory");
  else
    commit(bar);
}
template <bool PAIR>
__device__ __forceinline__ void take_tmem(u32 to_smem, u32 columns) {
  if (PAIR) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(to_smem), "r"(columns) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
  } else {
    tmem_alloc(to_smem, columns);
  }
}
template <bool PAIR>
__device__ __forceinline__ void leave_tmem(u32 at, u32 columns) {
  if (PAIR) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(at), "r"(columns));
  else tmem_free(at, columns);
}

// ---- tiles.  The grid has a block (or pair) for each; those that run take over the tiles of those that have not begun, one after the other.  (SMs' clocks
// differ when power is short, by a third between the slowest and the fastest seen: with tiles dealt out beforehand
// 16384 tokens, 8192 to 32768 columns, took 7.6 ms instead of 5.7.)
template <bool PAIR>
__device__ __forceinline__ void ask_for_tile(u32 to, u32 bar) {
  if (PAIR)
    asm volatile("clusterlaunchcontrol.try_cancel.async.shared::cta.mbarrier::complete_tx::bytes.multicast::cluster::all.b128 [%0], [%1];" ::"r"(to), "r"(bar) : "memory");
  else
    asm volatile("clusterlaunchcontrol.try_cancel.async.shared::cta.mbarrier::complete_tx::bytes.b128 [%0], [%1];" ::"r"(to), "r"(bar) : "memory");
}
// the answer's first block, or none
__device__ __forceinline__ bool answered(u32 at, u32& block) {
  u32 taken;
  asm volatile(
      "{\n\t.reg .pred p;\n\t.reg .b128 r;\n\t.reg .b32 y, z, w;\n\tld.shared.b128 r, [%2];\n\t"
      "clusterlaunchcontrol.query_cancel.is_canceled.pred.b128 p, r;\n\tselp.u32 %0, 1, 0, p;\n\tmov.u32 %1, 0;\n\t"
      "@p clusterlaunchcontrol.query_cancel.get_first_ctaid.v4.b32.b128 {%1, y, z, w}, r;\n\t}"
      : "=r"(taken), "=r"(block) : "r"(at) : "memory");
  fence_async();                                    // (read before the next answer is written)
  return taken != 0;
}
__device__ __forceinline__ void expect_at(u32 bar, u32 bytes, u32 rank) {
  asm volatile("{\n\t.reg .b32 a;\n\tmapa.shared::cluster.u32 a, %0, %2;\n\tmbarrier.arrive.expect_tx.release.cluster.shared::cluster.b64 _, [a], %1;\n\t}"
               ::"r"(bar), "r"(bytes), "r"(rank) : "memory");
}

// Tiles in the order in which blocks take them: bands of BAND tiles of rows, in a band column by column, so that the tiles
// that are summed at a time share their operands in the L2.
constexpr u32 BAND = 8;
struct Tile {
  u32 m, n, part;
};
__device__ __forceinline__ Tile tile_at(const Product& p, u32 t) {
  const u32 all = p.m_tiles * p.n_tiles, part = t / all;
  t -= part * all;
  const u32 band = t / (BAND * p.n_tiles), rest = t - band * BAND * p.n_tiles, height = min(BAND, p.m_tiles - band * BAND);
  return {band * BAND + rest % height, rest / height, part};
}

__device__ __forceinline__ uint4 read16(u32 at) {
  uint4 v;
  asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at) : "memory");
  return v;
}
__device__ __forceinline__ void write16(u32 at, u32 a, u32 b, u32 c, u32 d) {
  asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}
// 32 columns of a lane's row in a buffer: in 16-byte pieces that are permuted by the row as the copies do it
template <class E>
__device__ __forceinline__ u32 piece_at(u32 row, int column, int i) {
  const u32 piece = (u32)(column * (int)sizeof(E) / 16 + i);
  return row * 128 + ((piece ^ (row & 7)) << 4);
}
template <class E>
__device__ __forceinline__ void read32(u32 buffer, u32 row, int column, float (&v)[32]) {
  constexpr int N = 16 / sizeof(E);
#pragma unroll
  for (int i = 0; i < 32 / N; ++i) {
    const uint4 w = read16(buffer + piece_at<E>(row, column, i));
    Pack<E, N> p;
    p.w[0] = w.x, p.w[1] = w.y, p.w[2] = w.z, p.w[3] = w.w;
    float f[N];
    p.widen(f);
#pragma unroll
    for (int e = 0; e < N; ++e) v[i * N + e] = f[e];
  }
}
template <class E>
__device__ __forceinline__ void write32(u32 buffer, u32 row, int column, const float (&v)[32]) {
  constexpr int N = 16 / sizeof(E);
#pragma unroll
  for (int i = 0; i < 32 / N; ++i) {
    float f[N];
#pragma unroll
    for (int e = 0; e < N; ++e) f[e] = v[i * N + e];
    Pack<E, N> p;
    p.narrow(f);
    write16(buffer + piece_at<E>(row, column, i), p.w[0], p.w[1], p.w[2], p.w[3]);
  }
}

// A store of a box ends at the matrix's last column, but writes 16 bytes at least: where the last column is within them, a lane stores its row from the
// buffer itself.
template <class E>
__device__ __forceinline__ void store_edge(const ps_matrix& m, u32 row, u32 column, u32 rows, u32 columns, u32 buffer) {
  constexpr u32 N = 16 / sizeof(E);
  const u32 lane = threadIdx.x % 32;
  if (row + lane >= rows) return;
  E* const to = (E*)m.data + (u64)(row + lane) * m.stride + column;
#pragma unroll
  for (u32 i = 0; i < 8; ++i) {
    const uint4 w = read16(buffer + piece_at<E>(lane, 0, i));
    if (column + (i + 1) * N <= columns) {
      *reinterpret_cast<uint4*>(to + i * N) = w;
    } else {
      const u32 words[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
      for (u32 e = 0; e < N; ++e)
        if (column + i * N + e < columns) {
          if constexpr (sizeof(E) == 4) reinterpret_cast<u32*>(to)[i * N + e] = words[e];
          else reinterpret_cast<unsigned short*>(to)[i * N + e] = (unsigned short)(words[e / 2] >> (16 * (e % 2)));
        }
    }
  }
}

struct Maps {
  CUtensorMap a, b, out, residual, more, low;   // more: pre, written, or below, read; low: a's second part
};

// One product, or two that do not need one another: the tiles of one follow those of the other, whose are the longer ones, so that no SM
// waits for the end of a product while there is another.  (5003 tokens, 1416 to 2503 columns, dPre in two parts: 128 us by two
// kernels, 98 by one.  Started early by a programmatic launch, the second kernel took SMs from the first before its tiles were done: 200.)
struct None {};
template <class F, class G>
__global__ void __launch_bounds__(THREADS, 1) k_products(const __grid_constant__ Maps maps_f, const __grid_constant__ Maps maps_g, const Product of_f,
                                                        const Product of_g) {
  typedef typename F::T T;
  constexpr bool PAIR = F::PAIR, BOTH = !std::is_same<G, None>::value;
  constexpr int STAGES = F::STAGES;
  // `f` for the product that a tile belongs to
  const auto at_tile = [&](u32 t, const auto& f) {
    if constexpr (BOTH) {
      static_assert(F::STAGE == G::STAGE && F::COLUMNS == G::COLUMNS && F::PAIR == G::PAIR, "one ring, one shape");
      const u32 f_begins = of_f.after ? of_g.tiles : 0, g_begins = of_f.after ? 0 : of_f.tiles;
      if (of_f.after ? t < of_g.tiles : t >= of_f.tiles) return f(G{}, maps_g, of_g, t - g_begins);
      return f(F{}, maps_f, of_f, t - f_begins);
    } else {
      return f(F{}, maps_f, of_f, t);
    }
  };
  extern __shared__ unsigned char raw[];
  const u32 base = (smem_address(raw) + 1023u) & ~1023u;
  const u32 ring = base, buffers = ring + STAGES * F::STAGE, biases = buffers + F::BUFFERS, bars = biases + WRITERS * 128;
  // barriers: full and empty of each stage, full and empty of each sum, a writer's input
  const auto full = [&](int s) { return bars + 8 * s; };
  const auto empty = [&](int s) { return bars + 8 * (STAGES + s); };
  const auto sum_full = [&](int s) { return bars + 8 * (2 * STAGES + s); };
  const auto sum_empty = [&](int s) { return bars + 8 * (2 * STAGES + 2 + s); };
  const auto input = [&](int w) { return bars + 8 * (2 * STAGES + 4 + w); };
  const auto tile_full = [&](u32 n) { return bars + 8 * (2 * STAGES + 4 + WRITERS + n % TILES_AHEAD); };
  const auto tile_empty = [&](u32 n) { return bars + 8 * (2 * STAGES + 4 + WRITERS + TILES_AHEAD + n % TILES_AHEAD); };
  const auto answer = [&](u32 n) { return bars + 256 + 16 * (n % TILES_AHEAD); };
  const u32 wanted = bars + 256 + 16 * TILES_AHEAD;         // a tile's copies are nearly done: the next one may be asked for
  __shared__ u32 tmem_at;
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  const u32 rank = PAIR ? cluster_rank() : 0;

  if (threadIdx.x == 0) {
    for (int s = 0; s < STAGES; ++s) barrier_init(full(s), 1), barrier_init(empty(s), 1);
    for (int s = 0; s < 2; ++s) barrier_init(sum_full(s), 1), barrier_init(sum_empty(s), WRITERS * (PAIR ? 2 : 1));
    for (int w = 0; w < WRITERS; ++w) barrier_init(input(w), 1);
    for (u32 n = 0; n < TILES_AHEAD; ++n) barrier_init(tile_full(n), 1), barrier_init(tile_empty(n), PAIR ? 2 * WRITERS + 4 : WRITERS + 3);
    barrier_init(wanted, 1);
    fence_barrier_init();
  }
  if (warp == MMA_WARP) take_tmem<PAIR>(smem_address(&tmem_at), F::TMEM);
  fence_before();
  __syncthreads();
  if (PAIR) cluster_sync();
  fence_after();
  const u32 tmem = tmem_at;

  const u32 first = PAIR ? blockIdx.x / 2 : blockIdx.x;
  Waiter waiter(of_f.status);
  // a role's n-th answer: the tile to go on with, or none.  `speaks`: the thread that says that it has been read
  const auto next_tile = [&](u32 n, u32& t, bool speaks) {
    waiter.template wait<PAIR>(tile_full(n), (n / TILES_AHEAD) & 1);
    u32 block = 0;
    const bool more = !waiter.dead && answered(answer(n), block);
    t = PAIR ? block / 2 : block;
    if (speaks) {
      if (PAIR) arrive_at_leader(tile_empty(n));
      else barrier_arrive(tile_empty(n));
    }
    return more;
  };

  if (warp == COPY_WARP) {
    if (elected()) {
      u32 turn = 0;                                 // stages filled so far
      u32 count = 0, t = first;
      const auto copy = [&](auto form, const Maps& maps, const Product& p, u32 t) {
        typedef decltype(form) X;
        const Tile tile = tile_at(p, t);
        const int row = (int)(tile.m * (PAIR ? 256 : 128) + rank * ROWS), column = (int)(tile.n * F::COLUMNS + rank * F::B_ROWS);
        const u32 last = min((tile.part + 1) * p.steps_each, p.steps);
        u32 left = (last - tile.part * p.steps_each) * (X::TWO ? 2 : 1);
        const u32 ask = min(left, ASK_BEFORE);
        for (u32 begin = tile.part * p.steps_each; begin < last && !waiter.dead; begin += p.steps_at_once) {
#pragma unroll 1
          for (int low = X::TWO ? 1 : 0; low >= 0; --low)
            for (u32 k = begin, end = min(begin + p.steps_at_once, last); k < end; ++k, ++turn) {
              if (left-- == ask && rank == 0) barrier_arrive(wanted);
              const int s = turn % STAGES;
              waiter.template wait<PAIR>(empty(s), (turn / STAGES + 1) & 1);
              if (waiter.dead) break;
              if (rank == 0) barrier_expect(full(s), (PAIR ? 2 : 1) * p.stage_bytes);
              const u32 a = ring + s * F::STAGE, b = a + F::A_BYTES;
              const CUtensorMap* const a_map = low ? &maps.low : &maps.a;
              const int at = (int)(k * STEP);
              if (X::A_ACROSS) {
#pragma unroll
                for (int i = 0; i < ROWS / 64; ++i) load_box<PAIR>(a + i * ACROSS_PANEL, a_map, row + 64 * i, at, full(s));
              } else {
                load_box<PAIR>(a, a_map, at, row, full(s));
              }
              if (X::B_ACROSS) {
#pragma unroll
                for (int i = 0; i < X::B_LOADED / 64; ++i) load_box<PAIR>(b + i * ACROSS_PANEL, &maps.b, column + 64 * i, at, full(s));
              } else {
                load_box<PAIR>(b, &maps.b, at, column, full(s));
              }
            }
        }
      };
      do at_tile(t, copy);
      while (!waiter.dead && next_tile(count++, t, true));
      if (rank == 0) {                              // leave no copy in flight, also where a wait has run out
        Waiter last(of_f.status);
        for (u32 i = turn > STAGES ? turn - STAGES : 0; i < turn; ++i) last.template wait<PAIR>(full(i % STAGES), (i / STAGES) & 1);
      }
    }
    __syncwarp();
  } else if (warp == MMA_WARP) {
    if (rank == 0 && elected()) {
      u32 turn = 0, count = 0, sums = 0, t = first;
      const auto sum_up = [&](auto form, const Maps&, const Product& p, u32 t) {
        typedef decltype(form) X;
        constexpr u32 ins = instruction_of<X>();
        const u32 part = tile_at(p, t).part, last = min((part + 1) * p.steps_each, p.steps);
        for (u32 begin = part * p.steps_each; begin < last && !waiter.dead; begin += p.steps_at_once, ++sums) {
          const u32 end = min(begin + p.steps_at_once, last), d = tmem + (sums & 1) * F::SUM;
          waiter.template wait<PAIR>(sum_empty(sums & 1), (sums / 2 + 1) & 1);
          fence_after();
#pragma unroll 1
          for (int low = X::TWO ? 1 : 0; low >= 0; --low)
            for (u32 k = begin; k < end && !waiter.dead; ++k, ++turn) {
              const int s = turn % STAGES;
              waiter.template wait<PAIR>(full(s), (turn / STAGES) & 1);
              if (waiter.dead) break;
              fence_after();
              const u32 a = descriptor<X::A_ACROSS>(ring + s * F::STAGE), b = descriptor<X::B_ACROSS>(ring + s * F::STAGE + F::A_BYTES);
#pragma unroll
              for (int i = 0; i < STEP / 16; ++i) {
                if (X::TWO && i == 0 && low == 0 && k == begin) multiply_scaled<PAIR>(d, a, b, ins);
                else multiply<PAIR>(d, a + step_of<X::A_ACROSS>(i), b + step_of<X::B_ACROSS>(i), ins, k > begin || i > 0);
              }
              commit_to<PAIR>(empty(s));
            }
          if (!waiter.dead) commit_to<PAIR>(sum_full(sums & 1));
        }
      };
      do at_tile(t, sum_up);
      while (!waiter.dead && next_tile(count++, t, true));
    }
    __syncwarp();
  } else if (warp == TILE_WARP) {
    if (rank == 0 && elected()) {
      u32 t;
      for (u32 n = 0; !waiter.dead; ++n) {
        waiter.template wait<PAIR>(tile_empty(n), (n / TILES_AHEAD + 1) & 1);
        waiter.wait(wanted, n & 1);
        if (waiter.dead) break;
        if (PAIR) expect_at(tile_full(n), 16, 0), expect_at(tile_full(n), 16, 1);
        else barrier_expect(tile_full(n), 16);
        ask_for_tile<PAIR>(answer(n), tile_full(n));
        if (!next_tile(n, t, true)) break;
      }
    }
    __syncwarp();
  } else {
    const u32 mine = buffers + warp * 2 * BUFFER, other = mine + BUFFER;       // result and residual; pre or below
    const u32 bias_at = biases + warp * 128;
    const int quarter = warp % 4, half = warp / 4;
    u32 count = 0, sums = 0, inputs = 0, t = first;
    bool more = true;
    const auto write = [&](auto form, const Maps& maps, const Product& p, u32 t) {
      typedef decltype(form) X;
      typedef typename X::O O;
      constexpr int CHUNK = X::CHUNK;
      const Tile tile = tile_at(p, t);
      const u32 last = min((tile.part + 1) * p.steps_each, p.steps);
      const int row = (int)(tile.m * (PAIR ? 256 : 128) + rank * ROWS + quarter * 32);
      for (u32 begin = tile.part * p.steps_each; begin < last; begin += p.steps_at_once, ++sums) {
        // what is added to: the residual, or what this very warp has written of the sum so far
        const bool further = sizeof(O) == 4 && begin > tile.part * p.steps_each;
        const bool adds = p.has_residual || further;
        bool waited = false;
#pragma unroll 1
        for (int c = half; c < F::COLUMNS / CHUNK; c += 2) {
          const int column = (int)(tile.n * F::COLUMNS + c * CHUNK);
          if (row >= (int)p.m || column >= (int)p.n || waiter.dead) continue;
          const bool reads = adds || (X::KIND == INPUT_GRAD && p.has_below);
          if (lane == 0) {
            if (further) {
              wait_stores_done();
              asm volatile("fence.proxy.async;" ::: "memory");
            }
            wait_stores_read();                       // the buffers' last results have left
            if (reads) {
              barrier_expect(input(warp), ((adds ? 1 : 0) + (X::KIND == INPUT_GRAD && p.has_below ? 1 : 0)) * BUFFER);
              if (adds) load_rows(mine, further ? &maps.out : &maps.residual, column, row, further ? (int)tile.part : 0, input(warp));
              if (X::KIND == INPUT_GRAD && p.has_below) load_rows(other, &maps.more, column, row, 0, input(warp));
            }
          }
          if (X::KIND == OUTPUT && p.bias) {
#pragma unroll
            for (int i = lane; i < CHUNK; i += 32) {
              const unsigned short v = column + i < (int)p.n ? ((const unsigned short*)p.bias)[column + i] : (unsigned short)0;
              asm volatile("st.shared.u16 [%0], %1;" ::"r"(bias_at + 2 * i), "h"(v) : "memory");
            }
          }
          __syncwarp();
          if (!waited) {
            waiter.template wait<PAIR>(sum_full(sums & 1), (sums / 2) & 1);
            fence_after();
            waited = true;
          }
          if (reads) waiter.wait(input(warp), inputs++ & 1);
          waiter.dead = __any_sync(0xffffffffu, waiter.dead);      // (the lanes go on together)
          if (waiter.dead) continue;
#pragma unroll
          for (int h = 0; h < CHUNK; h += 32) {
            u32 sum[32];
            tmem_load32(sum, tmem + ((u32)(quarter * 32) << 16) + (sums & 1) * F::SUM + c * CHUNK + h);
            wait_loads();
            float v[32];
#pragma unroll
            for (int e = 0; e < 32; ++e) v[e] = __uint_as_float(sum[e]);
            if (X::KIND == OUTPUT) {
              if (p.bias)
#pragma unroll
                for (int e = 0; e < 32; e += 8) {
                  const uint4 w = read16(bias_at + 2 * (h + e));
                  Pack<T, 8> b;
                  b.w[0] = w.x, b.w[1] = w.y, b.w[2] = w.z, b.w[3] = w.w;
                  float f[8];
                  b.widen(f);
#pragma unroll
                  for (int i = 0; i < 8; ++i) v[e + i] += f[i];
                }
              if (p.has_pre) write32<T>(other, lane, h, v);
              activate(p.activation, v);
            }
            float f[32];
            if (X::KIND == INPUT_GRAD && p.has_below) {
              read32<T>(other, lane, h, f);
              times_slope(p.below_activation, v, f);
            }
            if (adds) {
              read32<O>(mine, lane, h, f);
#pragma unroll
              for (int e = 0; e < 32; ++e) v[e] += f[e];
            }
            write32<O>(mine, lane, h, v);
          }
          if (p.out.data && column + CHUNK > (int)p.n) {
            store_edge<O>(p.out, row, column, p.m, p.n, mine);
            if (X::KIND == OUTPUT && p.has_pre) store_edge<T>(p.pre, row, column, p.m, p.n, other);
            // The next copy into the buffers comes behind what the lanes have read and written there; a sum in 32 bits is read from memory again, too.
            if (sizeof(O) == 4) asm volatile("fence.proxy.async;" ::: "memory");
            else fence_async();
            __syncwarp();
            continue;
          }
          fence_async();
          __syncwarp();
          if (lane == 0) {
            store_rows(&maps.out, column, row, (int)tile.part, mine);
            if (X::KIND == OUTPUT && p.has_pre) store_rows(&maps.more, column, row, 0, other);
            commit_stores();
          }
        }
        if (!waited) {                                // (nothing of this tile is this warp's: it says so in turn all the same)
          waiter.template wait<PAIR>(sum_full(sums & 1), (sums / 2) & 1);
          fence_after();
        }
        waiter.dead = __any_sync(0xffffffffu, waiter.dead);
        fence_before();
        __syncwarp();
        if (lane == 0) {
          if (PAIR) arrive_at_leader(sum_empty(sums & 1));
          else barrier_arrive(sum_empty(sums & 1));
        }
      }
    };
    do {
      at_tile(t, write);
      more = !waiter.dead && next_tile(count, t, false);
      more = __all_sync(0xffffffffu, more);
      if (lane == 0) {                              // (all lanes have read it)
        if (PAIR) arrive_at_leader(tile_empty(count));
        else barrier_arrive(tile_empty(count));
      }
      ++count;
    } while (more);
    if (lane == 0) wait_stores_done();
    __syncwarp();
  }
  fence_before();
  __syncthreads();
  if (PAIR) cluster_sync();                         // neither block leaves while the other's products read its memory
  fence_after();
  if (warp == MMA_WARP) leave_tmem<PAIR>(tmem, F::TMEM);
}

// ---- dW out of the parts of a sum that was cut: parts[splits][m][pitch], added in order
template <class O>
__global__ void __launch_bounds__(256) k_join_parts(const float* parts, u32 splits, u64 m, u32 n, u32 pitch, O* out, u64 stride, u32 accumulate) {
  let_next_begin();
  wait_for_earlier();
  const u32 c = blockIdx.x * 256 + threadIdx.x;
  if (c >= n) return;
  for (u64 r = blockIdx.y; r < m; r += gridDim.y) {
    float sum = 0.f;
#pragma unroll 4
    for (u32 s = 0; s < splits; ++s) sum += parts[(s * m + r) * pitch + c];
    O* const to = out + r * stride + c;
    *to = narrow<O>(sum + (accumulate ? widen(*to) : 0.f));
  }
}

// ---- dPre = dY o act'(pre), rounded, and where `low` is given what the rounding took, 2^LOW_SHIFT times as large; and its sums by columns.  A lane has N
// columns, 8 or, where there are few rows and so few blocks, 2; a block 16 rows at a time.  A chunk of the rows leaves its sums in parts, the only one
// in `out`.  (ACT is PS_ACT_NONE for the sums alone.  With an activation and 8 columns a lane the 64 registers of two blocks an SM do not do: 84 to 104 bytes spill.  5003 x
// 2503 of half with silu and a low part take 35 us, of which the bytes are 15: 22 % of the memory's rate, issue slots 61 %.)
constexpr int SLOPE_WARPS = 16;
template <class T, int N, int ACT>
__global__ void __launch_bounds__(SLOPE_WARPS * 32, 2) k_slope(const ps_matrix d_y, const ps_matrix pre, const ps_matrix d_pre, const ps_matrix low, u64 rows, u32 cols,
                                                           u64 rows_each, float* parts, void* out, u32 out_wide, u32 accumulate) {
  constexpr int COLUMNS = 32 * N, AT_ONCE = N == 8 ? 4 : 8;
  __shared__ float sums[SLOPE_WARPS][COLUMNS];
  const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
  const u32 column = blockIdx.x * COLUMNS + lane * N;
  const int here = column >= cols ? 0 : (int)min((u32)N, cols - column);
  const u64 begin = blockIdx.y * rows_each, end = begin + rows_each < rows ? begin + rows_each : rows;
  float sum[N] = {};
  const auto load = [&](const T* from, Pack<T, N>& p) {
    p.clear();
    if (here == N) p.load(from);
    else
#pragma unroll
      for (int e = 0; e < N; ++e)
        if (e < here) p.w[e / 2] |= (u32)*reinterpret_cast<const unsigned short*>(from + e) << (16 * (e % 2));
  };
  const auto store = [&](T* to, const Pack<T, N>& p) {
    if (here == N) p.store(to);
    else
#pragma unroll
      for (int e = 0; e < N; ++e)
        if (e < here) reinterpret_cast<unsigned short*>(to)[e] = (unsigned short)(p.w[e / 2] >> (16 * (e % 2)));
  };
  if (here > 0)
    for (u64 first = begin + warp; first < end; first += AT_ONCE * SLOPE_WARPS) {
      Pack<T, N> g[AT_ONCE], at[AT_ONCE];
#pragma unroll
      for (int u = 0; u < AT_ONCE; ++u) {
        const u64 r = first + u * SLOPE_WARPS;
        g[u].clear();
        if (r < end) {
          load((const T*)d_y.data + r * d_y.stride + column, g[u]);
          if (ACT) load((const T*)pre.data + r * pre.stride + column, at[u]);
        }
      }
#pragma unroll
      for (int u = 0; u < AT_ONCE; ++u) {
        const u64 r = first + u * SLOPE_WARPS;
        float v[N], x[N];
        g[u].widen(v);
        if (ACT && r < end) {
          at[u].widen(x);
#pragma unroll
          for (int e = 0; e < N; ++e) v[e] *= slope<ACT>(x[e]);
          g[u].narrow(v);
          store((T*)d_pre.data + r * d_pre.stride + column, g[u]);
          if (low.data) {
            g[u].widen(x);
#pragma unroll
            for (int e = 0; e < N; ++e) x[e] = (v[e] - x[e]) * (float)(1 << LOW_SHIFT);
            g[u].narrow(x);
            store((T*)low.data + r * low.stride + column, g[u]);
          }
        }
#pragma unroll
        for (int e = 0; e < N; ++e) sum[e] += v[e];
      }
    }
  if (parts == nullptr && out == nullptr) return;
#pragma unroll
  for (int e = 0; e < N; ++e) sums[warp][lane * N + e] = sum[e];
  __syncthreads();
  const u32 c = blockIdx.x * COLUMNS + threadIdx.x;
  if (threadIdx.x >= COLUMNS || c >= cols) return;
  float all[4] = {};
#pragma unroll
  for (int w = 0; w < SLOPE_WARPS; ++w) all[w % 4] += sums[w][threadIdx.x];
  const float total = (all[0] + all[1]) + (all[2] + all[3]);
  if (parts) {
    parts[(u64)blockIdx.y * cols + c] = total;
  } else if (out_wide) {
    float* const to = (float*)out + c;
    *to = accumulate ? *to + total : total;
  } else {
    T* const to = (T*)out + c;
    *to = narrow<T>(accumulate ? widen(*to) + total : total);
  }
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
// a matrix as boxes of 128 bytes by `box_rows`; as one of `parts` matrices behind one another where it is written or read by warps
template <class E>
bool encode(CUtensorMap& map, u32 dtype, const ps_matrix& m, u64 rows, u64 cols, u32 box_rows, u32 parts) {
  const cuuint64_t stride = rows > 1 ? m.stride * sizeof(E) : (cols * sizeof(E) + 15) / 16 * 16;
  const cuuint64_t extents[3] = {cols, rows, parts ? parts : 1}, strides[2] = {stride, stride * rows};
  const cuuint32_t box[3] = {(cuuint32_t)(128 / sizeof(E)), box_rows, 1}, steps[3] = {1, 1, 1};
  const CUtensorMapDataType type = sizeof(E) == 4 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32
                                   : dtype == PS_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16;
  return encoder()(&map, type, parts ? 3 : 2, m.data, extents, strides, box, steps, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                   CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

constexpr ps_matrix NOTHING = {nullptr, 0};

// C[m][n] = sum over k of A B, and what is done with it
struct Call {
  Kind kind;
  ps_matrix a, b, out, residual, more;
  u64 m, n, k;
  u32 parts;                              // of the sum, stored one behind the other
  const void* bias;
  u32 activation, below_activation;
  ps_matrix low;                          // a's second part (WEIGHT_GRAD_TWO)
};

// what a kernel is told of a product; one without a result has no tiles
template <class F>
bool describe(u32 dtype, const Call& c, volatile u32* status, Maps& maps, Product& p) {
  typedef typename F::T T;
  typedef typename F::O O;
  p.status = status;
  if (!c.out.data) return true;
  p.m = (u32)c.m, p.n = (u32)c.n, p.steps = (u32)((c.k + STEP - 1) / STEP);
  p.m_tiles = (u32)((c.m + (F::PAIR ? 255 : 127)) / (F::PAIR ? 256 : 128));
  p.n_tiles = (u32)((c.n + F::COLUMNS - 1) / F::COLUMNS);
  p.steps_each = (p.steps + c.parts - 1) / c.parts;
  p.splits = (p.steps + p.steps_each - 1) / p.steps_each;
  p.steps_at_once = sizeof(O) == 4 ? STEPS_AT_ONCE : p.steps_each;
  p.bias = c.bias;
  p.activation = c.activation, p.below_activation = c.below_activation;
  p.has_residual = c.residual.data != nullptr;
  p.has_below = F::KIND == INPUT_GRAD && c.more.data;
  p.has_pre = F::KIND == OUTPUT && c.more.data;
  if (c.n % (16 / sizeof(O)) && c.parts == 1) {            // (the parts' rows are whole 16 bytes)
    p.out = c.out;
    if (p.has_pre) p.pre = c.more;
  }
  // Boxes have no more rows than the matrix (in eights): a copy takes its time for rows that are not there as well.  (What then stands in the
  // rest of a tile in shared memory becomes results that are not stored.  A token, 8192 to 8192 columns: 33 us, with boxes of 128 rows 56.)
  const auto box_rows = [](u64 rows, u32 most) { return (u32)std::min<u64>((rows + 7) / 8 * 8, most); };
  const u32 a_rows = F::A_ACROSS ? STEP : box_rows(c.m, ROWS), b_rows = F::B_ACROSS ? STEP : box_rows(c.n, F::B_ROWS);
  p.stage_bytes = (F::A_ACROSS ? F::A_BYTES : a_rows * 128) + (F::B_ACROSS ? F::B_BYTES : b_rows * 128);
  bool ok = F::A_ACROSS ? encode<T>(maps.a, dtype, c.a, c.k, c.m, a_rows, 0) : encode<T>(maps.a, dtype, c.a, c.m, c.k, a_rows, 0);
  ok = ok && (F::B_ACROSS ? encode<T>(maps.b, dtype, c.b, c.k, c.n, b_rows, 0) : encode<T>(maps.b, dtype, c.b, c.n, c.k, b_rows, 0));
  ok = ok && encode<O>(maps.out, dtype, c.out, c.m, c.n, 32, c.parts);
  if (F::TWO) ok = ok && encode<T>(maps.low, dtype, c.low, c.k, c.m, STEP, 0);
  if (p.has_residual) ok = ok && encode<O>(maps.residual, dtype, c.residual, c.m, c.n, 32, 1);
  if (c.more.data) ok = ok && encode<T>(maps.more, dtype, c.more, c.m, c.n, 32, 1);
  const u64 tiles = (u64)p.m_tiles * p.n_tiles * p.splits;
  p.tiles = (u32)tiles;
  return ok && tiles < (1u << 29);
}

template <class F, class G>
cudaError_t launch_products(u32 dtype, const Call& f, const Call* g, volatile u32* status, cudaStream_t stream) {
  Maps maps[2] = {};
  Product p[2] = {};
  if (!describe<F>(dtype, f, status, maps[0], p[0])) return cudaErrorInvalidValue;
  if constexpr (!std::is_same<G, None>::value)
    if (!describe<G>(dtype, *g, status, maps[1], p[1])) return cudaErrorInvalidValue;
  static std::atomic<u64> prepared{0};                      // devices on which the kernel's shared memory has been asked for
  int device;
  cudaError_t e = cudaGetDevice(&device);
  if (e != cudaSuccess) return e;
  if (device >= 64 || !(prepared.load() >> device & 1)) {
    e = cudaFuncSetAttribute(k_products<F, G>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)F::SMEM);
    if (e != cudaSuccess) return e;
    if (device < 64) prepared |= (u64)1 << device;
  }
  const u32 tiles = p[0].tiles + p[1].tiles;
  p[0].after = (u64)p[1].steps_each > (u64)p[0].steps_each * (F::TWO ? 2 : 1);
  cudaLaunchAttribute pair;
  pair.id = cudaLaunchAttributeClusterDimension;
  pair.val.clusterDim.x = 2, pair.val.clusterDim.y = pair.val.clusterDim.z = 1;
  cudaLaunchConfig_t config = {};
  config.gridDim = dim3(F::PAIR ? 2 * tiles : tiles);
  config.blockDim = dim3(THREADS);
  config.dynamicSmemBytes = F::SMEM;
  config.stream = stream;
  config.attrs = &pair;
  config.numAttrs = F::PAIR ? 1 : 0;
  return cudaLaunchKernelEx(&config, k_products<F, G>, maps[0], maps[1], p[0], p[1]);
}

// The tile's shape: the one with which the blocks are done first by what was measured of it, in cycles: for 64 steps of the sum, for writing a tile (of
// which the longer counts, tile after tile), and for a launch's beginning and end.
struct TileCost {
  u32 rows, columns;
  bool pair;
  u32 step, write, around;
};
constexpr TileCost TILE_COSTS[] = {{256, 256, true, 600, 3800, 13000}, {256, 192, true, 510, 3400, 12000}, {256, 128, true, 395, 1900, 11000},
                                   {128, 128, false, 450, 1500, 10500}, {128, 64, false, 320, 1400, 9500}};
// (Tiles are dealt out one by one: with two products, or none that a block gets more of than another, the blocks are done when their share is.)
int shape_for(const Call* const (&calls)[2], int sm_count) {
  int best = 0;
  u64 least = ~(u64)0;
  for (int i = 0; i < 5; ++i) {
    const TileCost& t = TILE_COSTS[i];
    const u64 at_once = t.pair ? sm_count / 2 : sm_count;
    u64 all = 0, longest = 0, shortest = ~(u64)0, count = 0;
    for (const Call* c : calls)
      if (c && c->out.data) {
        const u64 tiles = ((c->m + t.rows - 1) / t.rows) * ((c->n + t.columns - 1) / t.columns) * c->parts;
        const u64 steps = ((c->k + STEP - 1) / STEP + c->parts - 1) / c->parts * (c->kind == WEIGHT_GRAD_TWO ? 2 : 1);
        // (half of a tile of 192 columns that lie across the sum is loaded as 128)
        const u64 tile = std::max<u64>(steps * (i == 1 && c->kind != OUTPUT ? 640 : t.step), t.write);
        all += tiles * tile, count += tiles;
        longest = std::max(longest, tile), shortest = std::min(shortest, tile);
      }
    // one kind of tile: whole rounds; two: the share, and half of a short one more
    const u64 cost = (longest == shortest ? (count + at_once - 1) / at_once * longest : std::max(longest, (all + at_once - 1) / at_once + shortest / 2)) + t.around;
    if (cost < least) least = cost, best = i;
  }
  return best;
}
template <class T>
cudaError_t output(u32 dtype, const Call& c, volatile u32* status, int sm_count, cudaStream_t stream) {
  switch (shape_for({&c, nullptr}, sm_count)) {
    case 0: return launch_products<Form<T, T, OUTPUT, 256, true>, None>(dtype, c, nullptr, status, stream);
    case 1: return launch_products<Form<T, T, OUTPUT, 192, true>, None>(dtype, c, nullptr, status, stream);
    case 2: return launch_products<Form<T, T, OUTPUT, 128, true>, None>(dtype, c, nullptr, status, stream);
    case 3: return launch_products<Form<T, T, OUTPUT, 128, false>, None>(dtype, c, nullptr, status, stream);
    default: return launch_products<Form<T, T, OUTPUT, 64, false>, None>(dtype, c, nullptr, status, stream);
  }
}
template <class T, class O, Kind KIND>
cudaError_t gradients(u32 dtype, const Call& w, const Call& x, volatile u32* status, int sm_count, cudaStream_t stream) {
  switch (shape_for({&w, &x}, sm_count)) {
    case 0: return launch_products<Form<T, O, KIND, 256, true>, Form<T, T, INPUT_GRAD, 256, true>>(dtype, w, &x, status, stream);
    case 1: return launch_products<Form<T, O, KIND, 192, true>, Form<T, T, INPUT_GRAD, 192, true>>(dtype, w, &x, status, stream);
    case 2: return launch_products<Form<T, O, KIND, 128, true>, Form<T, T, INPUT_GRAD, 128, true>>(dtype, w, &x, status, stream);
    case 3: return launch_products<Form<T, O, KIND, 128, false>, Form<T, T, INPUT_GRAD, 128, false>>(dtype, w, &x, status, stream);
    default: return launch_products<Form<T, O, KIND, 64, false>, Form<T, T, INPUT_GRAD, 64, false>>(dtype, w, &x, status, stream);
  }
}

constexpr u64 SMS = 148;          // (what a sum's order depends on does not ask the device)

// parts of the sum over the tokens for dW: as many as bring tiles for all SMs, each of 16 stages at least
u32 weight_parts(const LinearArgs& a) {
  const u64 tiles = ((a.outputs + 127) / 128) * ((a.inputs + 127) / 128), steps = (a.tokens + STEP - 1) / STEP;
  const u64 parts = std::min(std::max<u64>(1, SMS / tiles), std::max<u64>(1, steps / 16));
  if (parts == 1) return 1;
  const u64 each = (steps + parts - 1) / parts;
  return (u32)((steps + each - 1) / each);
}
u64 up(u64 n, u64 to) { return (n + to - 1) / to * to; }
// Rows of a chunk for the sums by columns: all where there are few (a launch less), else as many as give each SM two blocks, in whole batches of a block.
constexpr u64 FEW_TOKENS = 512;
u64 slope_rows(const LinearArgs& a) {
  if (a.tokens <= FEW_TOKENS) return std::max<u64>(a.tokens, 1);
  const u64 across = (a.outputs + 255) / 256, chunks = std::max<u64>(1, 2 * SMS / across);
  return up((a.tokens + chunks - 1) / chunks, 4 * SLOPE_WARPS);
}
u64 slope_chunks(const LinearArgs& a) { return std::max<u64>(1, (a.tokens + slope_rows(a) - 1) / slope_rows(a)); }
// dPre's rows begin at multiples of 32 bytes: of rows that begin at 16 alone a box takes a fifth longer
u64 d_pre_stride(const LinearArgs& a) { return up(a.outputs, 16); }
struct Work {
  size_t low, sums, parts, all;           // (d_pre stands first)
};
Work work_of(const LinearArgs& a) {
  Work w;
  w.low = a.activation ? up(a.tokens * d_pre_stride(a) * 2, 256) : 0;
  w.sums = a.activation && a.grad_dtype == PS_F32 ? 2 * w.low : w.low;
  w.parts = w.sums + up(slope_chunks(a) * a.outputs * 4, 256);
  const u32 parts = weight_parts(a);
  w.all = w.parts + (parts > 1 ? parts * a.outputs * up(a.inputs, 4) * 4 : 0);
  return w;
}

template <class T>
cudaError_t forward(const LinearArgs& a, int sm_count, cudaStream_t stream) {
  Call c = {OUTPUT, a.x, a.weight, a.y, a.residual, a.pre, a.tokens, a.outputs, a.inputs, 1, a.bias, a.activation, 0, NOTHING};
  return output<T>(a.dtype, c, a.status, sm_count, stream);
}

template <class T>
cudaError_t backward(const LinearArgs& a, int sm_count, cudaStream_t stream) {
  const Work where = work_of(a);
  char* const work = (char*)a.work;
  const u64 chunks = slope_chunks(a);
  float* const sums = a.d_bias && chunks > 1 ? (float*)(work + where.sums) : nullptr;
  ps_matrix d_pre = a.d_y, low = NOTHING;
  if (a.activation) d_pre = {work, d_pre_stride(a)};
  if (a.activation && a.grad_dtype == PS_F32 && a.d_weight.data) low = {work + where.low, d_pre_stride(a)};
  cudaError_t e = cudaSuccess;
  const auto slopes = [&] {
    const u64 each = slope_rows(a);
    const bool few = a.tokens <= FEW_TOKENS;
    const dim3 grid((u32)((a.outputs + (few ? 63 : 255)) / (few ? 64 : 256)), (u32)chunks);
    const u32 wide = a.grad_dtype == PS_F32;
    void* const out = chunks > 1 ? nullptr : a.d_bias;
    const auto go = [&](auto kernel) { kernel<<<grid, SLOPE_WARPS * 32, 0, stream>>>(a.d_y, a.pre, d_pre, low, a.tokens, (u32)a.outputs, each, sums, out, wide, a.accumulate); };
#define PS_EACH(ACT) \
  if (a.activation == ACT) go(few ? k_slope<T, 2, ACT> : k_slope<T, 8, ACT>);
    PS_EACH(PS_ACT_NONE) PS_EACH(PS_ACT_RELU) PS_EACH(PS_ACT_GELU) PS_EACH(PS_ACT_GELU_TANH) PS_EACH(PS_ACT_SILU)
#undef PS_EACH
    return cudaGetLastError();
  };
  if (a.activation) e = slopes();
  const u32 parts = weight_parts(a), pitch = (u32)up(a.inputs, 4);
  const bool wide = a.grad_dtype == PS_F32 || parts > 1;
  if (e == cudaSuccess && a.tokens && (a.d_x.data || a.d_weight.data)) {
    const Call x = {INPUT_GRAD, d_pre, a.weight, a.d_x, a.residual, a.below, a.tokens, a.inputs, a.outputs, 1, nullptr, 0, a.below_activation, NOTHING};
    Call w = {low.data ? WEIGHT_GRAD_TWO : WEIGHT_GRAD, d_pre, a.x, a.d_weight, a.accumulate ? a.d_weight : NOTHING, NOTHING, a.outputs, a.inputs, a.tokens, parts,
              nullptr, 0, 0, low};
    if (a.d_weight.data && parts > 1) w.out = {work + where.parts, pitch}, w.residual = NOTHING;
    e = !wide ? gradients<T, T, WEIGHT_GRAD>(a.dtype, w, x, a.status, sm_count, stream)
        : low.data ? gradients<T, float, WEIGHT_GRAD_TWO>(a.dtype, w, x, a.status, sm_count, stream)
                   : gradients<T, float, WEIGHT_GRAD>(a.dtype, w, x, a.status, sm_count, stream);
  } else if (e == cudaSuccess && a.d_weight.data && !a.accumulate) {
    const size_t width = a.grad_dtype == PS_F32 ? 4 : 2;
    e = cudaMemset2DAsync(a.d_weight.data, a.d_weight.stride * width, 0, a.inputs * width, a.outputs, stream);
  }
  if (e == cudaSuccess && a.d_weight.data && a.tokens && parts > 1) {
    const dim3 grid((u32)((a.inputs + 255) / 256), (u32)std::min<u64>(a.outputs, 65535));
    const float* const from = (const float*)(work + where.parts);
    if (a.grad_dtype == PS_F32) e = launch_next(k_join_parts<float>, grid, 256, 0, stream, from, parts, a.outputs, (u32)a.inputs, pitch, (float*)a.d_weight.data, a.d_weight.stride, a.accumulate);
    else e = launch_next(k_join_parts<T>, grid, 256, 0, stream, from, parts, a.outputs, (u32)a.inputs, pitch, (T*)a.d_weight.data, a.d_weight.stride, a.accumulate);
  }
  if (e == cudaSuccess && !a.activation && a.d_bias) e = slopes();
  if (e == cudaSuccess && sums) e = join_columns(a.grad_dtype, sums, (u32)chunks, 1, a.outputs, a.d_bias, nullptr, a.accumulate, stream);
  return e;
}

}  // namespace

cudaError_t launch_linear_forward(const LinearArgs& a, int sm_count, cudaStream_t stream) {
  if (!encoder()) return cudaErrorNotSupported;
  return a.dtype == PS_BF16 ? forward<__nv_bfloat16>(a, sm_count, stream) : forward<__half>(a, sm_count, stream);
}

size_t linear_backward_bytes(const LinearArgs& a) { return work_of(a).all; }

cudaError_t launch_linear_backward(const LinearArgs& a, int sm_count, cudaStream_t stream) {
  if (!encoder()) return cudaErrorNotSupported;
  return a.dtype == PS_BF16 ? backward<__nv_bfloat16>(a, sm_count, stream) : backward<__half>(a, sm_count, stream);
}
