// The embedding lookup and its gradient.
//
//   out[t]     = scale * table[token[t] - first_row]           (zeros where that row is not held)
//   d_table[v] = scale * sum over t with token[t] - first_row = v, t ascending, of d_out[t]
//
// Sums are held in 32 bits and rounded once.
//
// The gradient sorts (row, t) by row with t ascending (a stable radix sort of row numbers alone, or for few tokens a count, so nothing is left
// to the order in which blocks run), marks where each row's list begins and ends, and gives each row of the table to warps that
// sum its list: every row of d_table is written once (by few tokens twice where it has some), every row of d_out read once.  A list of c tokens is cut
// from its own beginning into pieces of 32 and pieces of 1024, which other blocks sum first; the warp adds the sums of
// the pieces of 1024, then of the pieces of 32 behind them, then the rest: at most c / 1024 + 62 terms (below 4096 tokens
// in all there are no pieces of 1024).  The cut follows from c and the number of tokens, so a row's bits are the same whatever other rows the
// table holds.
//
// What bounds them: bytes.  131072 lookups of 8192 bfloat16 in 128000 rows: 494 us, 5.7 TB/s by what has to move (words of middling frequency
// leave the L2 between two lookups and are read again).  The gradient of as many tokens into 256000 rows, 6.2 GB: 1.15 ms, 5.4 TB/s: 0.91 ms the
// rows (5.9 TB/s), 0.16 the pieces, 0.04 the sort, whose kernels are small.  2048 tokens into 32000 rows of 768: 18.8 us, a
// chain of three kernels of which the first writes the 49 MB of zeros.
#include "ps_train.cuh"

namespace {
using namespace train;

// the row of the table that token t looks up, or rows where none that is held
__device__ __forceinline__ u32 row_of(const EmbedArgs& a, u64 t) {
  const s64 id = a.token_bytes == 8 ? ((const s64*)a.tokens)[t] : (s64)((const int*)a.tokens)[t];
  const u64 row = (u64)id - a.first_row;
  return id >= 0 && (u64)id >= a.first_row && row < a.rows ? (u32)row : (u32)a.rows;
}

// ------------------------------------------------------------------ lookup
// A warp takes LOADS packs a lane of a token's row at a time, of 32 bytes where all rows begin at multiples of that.  (131072 lookups of 8192
// bfloat16 in 128000 rows: 494 us; with results that stay in the L2 506, with two packs 559, with four of 16 bytes 551.  More or fewer
// blocks an SM take longer: 560 with five, 548 with three.)
constexpr int LOOKUP_BLOCKS = 4;
template <class T, int N> constexpr int LOOKUP_LOADS = sizeof(T) * N == 32 ? 1 : 4;
template <class T, int N>
__global__ void __launch_bounds__(256, LOOKUP_BLOCKS) k_lookup(EmbedArgs a, u32 chunks, Divider by_chunk, u32 items) {
  constexpr bool WIDE = sizeof(T) * N == 32;
  constexpr int LOADS = LOOKUP_LOADS<T, N>;
  const u32 lane = threadIdx.x % 32, step = gridDim.x * 8;
  u32 item = blockIdx.x * 8 + threadIdx.x / 32, next = item < items ? row_of(a, by_chunk.of(item)) : 0;
  for (; item < items; item += step) {
    const u32 t = by_chunk.of(item), row = next;
    if (item + step < items) next = row_of(a, by_chunk.of(item + step));        // (the next one's, ahead)
    const u64 column = (u64)(item - t * chunks) * (32 * N * LOADS) + lane * N;
    Pack<T, N> v[LOADS];
    const T* from = (const T*)a.table + row * a.table_stride + column;
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
      v[i].clear();
      if (row < a.rows && column + i * 32 * N < a.dim) {
        if constexpr (WIDE) v[i].load32(from + i * 32 * N);
        else v[i].load(from + i * 32 * N);
      }
    }
    T* to = (T*)a.out + t * a.out_stride + column;
#pragma unroll
    for (int i = 0; i < LOADS; ++i)
      if (column + i * 32 * N < a.dim) {
        float x[N];
        v[i].widen(x);
#pragma unroll
        for (int e = 0; e < N; ++e) x[e] = row < a.rows ? x[e] * a.scale : 0.f;
        v[i].narrow(x);
        if constexpr (WIDE) v[i].store32_passing(to + i * 32 * N);
        else v[i].store_passing(to + i * 32 * N);
      }
  }
}

// ------------------------------------------------------------------ sort
constexpr int SORT_THREADS = 512, SORT_ITEMS = 4, SORT_TILE = SORT_THREADS * SORT_ITEMS, SORT_WARPS = SORT_THREADS / 32;
constexpr int MAX_BITS = 9, MAX_DIGITS = 1 << MAX_BITS;

struct SortArgs {
  u32 n, chunk, blocks;        // tokens, and how many of them in a row a block takes
  u32 shift, bits, passes;
  const u32 *keys_in, *values_in;   // null: the tokens themselves, and their places
  u32 *keys_out, *values_out;
  u32* counts;                 // [blocks][1 << bits]
};

__device__ __forceinline__ u32 key_at(const EmbedArgs& a, const u32* keys, u32 i) { return keys ? keys[i] : row_of(a, i); }

// exclusive sums of v over the block's threads (512)
__device__ __forceinline__ u32 scan_block(u32 v, u32* warp_sums) {
  const u32 lane = threadIdx.x % 32, warp = threadIdx.x / 32;
  u32 sum = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const u32 other = __shfl_up_sync(0xffffffffu, sum, o);
    if (lane >= (u32)o) sum += other;
  }
  if (lane == 31) warp_sums[warp] = sum;
  __syncthreads();
  if (warp == 0) {
    u32 w = lane < SORT_WARPS ? warp_sums[lane] : 0;
#pragma unroll
    for (int o = 1; o < SORT_WARPS; o <<= 1) {
      const u32 other = __shfl_up_sync(0xffffffffu, w, o);
      if (lane >= (u32)o) w += other;
    }
    if (lane < SORT_WARPS) warp_sums[lane] = w;
  }
  __syncthreads();
  return sum - v + (warp ? warp_sums[warp - 1] : 0);
}

static_assert(MAX_DIGITS == SORT_THREADS, "a thread a digit");
struct SortShared {
  u32 base[MAX_DIGITS];                   // where the block's next item of a digit goes
  u32 count[SORT_WARPS][MAX_DIGITS];
  u32 warp_sums[SORT_WARPS];
};

// Puts items [begin, end) in their places, base[digit] on.  A warp takes 32 * SORT_ITEMS items in a row; an item's rank among those of its
// digit is the number before it in the lanes, in the warp's earlier rounds and in the earlier warps.
__device__ void place_items(const EmbedArgs& a, const SortArgs& s, u32 begin, u32 end, SortShared& sh) {
  const u32 lane = threadIdx.x % 32, warp = threadIdx.x / 32, digits = 1u << s.bits;
  for (u32 tile = begin; tile < end; tile += SORT_TILE) {
#pragma unroll
    for (int w = 0; w < SORT_WARPS; ++w) sh.count[w][threadIdx.x] = 0;
    __syncthreads();
    u32 key[SORT_ITEMS], rank[SORT_ITEMS];
#pragma unroll
    for (int r = 0; r < SORT_ITEMS; ++r) {
      const u32 i = tile + warp * 32 * SORT_ITEMS + r * 32 + lane;
      key[r] = i < end ? key_at(a, s.keys_in, i) : 0;
    }
#pragma unroll
    for (int r = 0; r < SORT_ITEMS; ++r) {
      const bool there = tile + warp * 32 * SORT_ITEMS + r * 32 + lane < end;
      const u32 digit = there ? (key[r] >> s.shift) & (digits - 1) : digits;     // the absent ones are each other's
      const u32 same = __match_any_sync(0xffffffffu, digit), before = __popc(same & ((1u << lane) - 1));
      u32 had = 0;
      if (there) had = sh.count[warp][digit];
      __syncwarp();
      if (there && before == 0) sh.count[warp][digit] = had + __popc(same);
      __syncwarp();
      rank[r] = had + before;
    }
    __syncthreads();
    if (threadIdx.x < digits) {
      u32 sum = sh.base[threadIdx.x];
#pragma unroll
      for (int w = 0; w < SORT_WARPS; ++w) {
        const u32 c = sh.count[w][threadIdx.x];
        sh.count[w][threadIdx.x] = sum;
        sum += c;
      }
      sh.base[threadIdx.x] = sum;
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < SORT_ITEMS; ++r) {
      const u32 i = tile + warp * 32 * SORT_ITEMS + r * 32 + lane;
      if (i < end) {
        const u32 to = sh.count[warp][(key[r] >> s.shift) & (digits - 1)] + rank[r];
        s.keys_out[to] = key[r];
        s.values_out[to] = s.keys_in ? s.values_in[i] : i;
      }
    }
    __syncthreads();
  }
}

__global__ void __launch_bounds__(SORT_THREADS) k_sort_count(EmbedArgs a, SortArgs s) {
  __shared__ u32 count[MAX_DIGITS];
  let_next_begin();
  count[threadIdx.x] = 0;
  if (s.keys_in) wait_for_earlier();        // (the first pass reads tokens alone)
  __syncthreads();
  const u32 digits = 1u << s.bits, end = min(s.n, (blockIdx.x + 1) * s.chunk);
  for (u32 i = blockIdx.x * s.chunk + threadIdx.x; i < end; i += SORT_THREADS)
    atomicAdd(&count[(key_at(a, s.keys_in, i) >> s.shift) & (digits - 1)], 1u);
  __syncthreads();
  if (threadIdx.x < digits) s.counts[blockIdx.x * digits + threadIdx.x] = count[threadIdx.x];
}

__global__ void __launch_bounds__(SORT_THREADS) k_sort_place(EmbedArgs a, SortArgs s) {
  __shared__ SortShared sh;
  let_next_begin();
  wait_for_earlier();
  const u32 digits = 1u << s.bits;
  u32 before = 0, all = 0;
  if (threadIdx.x < digits) {
#pragma unroll 8
    for (u32 b = 0; b < s.blocks; ++b) {
      const u32 c = s.counts[b * digits + threadIdx.x];
      all += c;
      before += b < blockIdx.x ? c : 0;
    }
  }
  sh.base[threadIdx.x] = scan_block(all, sh.warp_sums) + before;
  place_items(a, s, blockIdx.x * s.chunk, min(s.n, (blockIdx.x + 1) * s.chunk), sh);
}

// Where a row's list begins and ends in the sorted order.  (The array is zeros before: a row without tokens has none.)
__global__ void __launch_bounds__(256) k_mark(const u32* keys, u32 n, uint2* ranges, u64 rows) {
  let_next_begin();
  wait_for_earlier();
  const u32 i = blockIdx.x * 256 + threadIdx.x;
  if (i >= n) return;
  const u32 key = keys[i];
  if (key >= rows) return;
  if (i == 0 || keys[i - 1] != key) ranges[key].x = i;
  if (i + 1 == n || keys[i + 1] != key) ranges[key].y = i + 1;
}

// Few tokens need no passes: a token's place is the number of smaller rows before or behind it plus the number of equal ones before it, and
// its row's list begins behind the smaller ones.  A warp counts for a token, over all rows in shared memory: n^2 comparisons on all
// SMs (2048 tokens: 6 us, most of it launch and loads, where one block's radix passes took 11).
//
// Few tokens leave most rows of the table without any.  Blocks behind those that count write zeros to all rows meanwhile, and
// the rows that have tokens are written again by k_lists.  (2048 tokens into 32000 rows of 768: 18.8 us in a loop, 27.6 with the L2 flushed
// before; 23.8 and 33.8 with k_gradient over all rows behind the places, and an array of lists to clear.  8192 into 128000 rows of 4096:
// 250 and 253, into 300 of 1024: 71 and 93, into 8000: 70 and 68.)
constexpr u32 RANK_MOST = 8192;
struct Fill {
  char* table;                 // null: nothing is to be cleared
  u64 units, stride;           // of a row: accesses of WIDTH bytes, and bytes from one to the next
  u32 rows;
};
template <int WIDTH> struct Unit { typedef uint4 type; };
template <> struct Unit<4> { typedef u32 type; };
template <> struct Unit<2> { typedef unsigned short type; };
template <int WIDTH>
__device__ __forceinline__ void fill(const Fill& f, u32 block, u32 blocks) {
  typedef typename Unit<WIDTH>::type U;
  // a row of so many accesses, or a part of it, to a block at a time
  constexpr u32 PART = 256 * 8;
  const u64 parts = (f.units + PART - 1) / PART;
  for (u64 i = block; i < f.rows * parts; i += blocks) {
    const u64 r = parts == 1 ? i : i / parts, first = (i - r * parts) * PART;
    U* const at = reinterpret_cast<U*>(f.table + r * f.stride) + first;
#pragma unroll
    for (u32 e = 0; e < 8; ++e)
      if (first + e * 256 + threadIdx.x < f.units) at[e * 256 + threadIdx.x] = U{};
  }
}
template <int WIDTH>
__global__ void __launch_bounds__(256) k_rank(EmbedArgs a, u32 n, u32* keys, u32* places, uint2* ranges, u32 counting, Fill f) {
  extern __shared__ uint4 rows4[];
  u32* const rows = reinterpret_cast<u32*>(rows4);
  let_next_begin();
  if (blockIdx.x >= counting) {
    fill<WIDTH>(f, blockIdx.x - counting, gridDim.x - counting);
    return;
  }
  const u32 lane = threadIdx.x % 32, fours = (n + 3) / 4;
  for (u32 i = threadIdx.x; i < fours * 4; i += 256) rows[i] = i < n ? row_of(a, i) : 0xffffffffu;
  __syncthreads();
  for (u32 t = blockIdx.x * 8 + threadIdx.x / 32; t < n; t += counting * 8) {
    const u32 key = rows[t];
    u32 less = 0, same = 0, before = 0;
    for (u32 i = lane; i < fours; i += 32) {
      const uint4 v = rows4[i];
      const u32 k[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
      for (u32 e = 0; e < 4; ++e) {
        less += k[e] < key;
        same += k[e] == key;
        before += k[e] == key && 4 * i + e < t;
      }
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      less += __shfl_xor_sync(0xffffffffu, less, o);
      same += __shfl_xor_sync(0xffffffffu, same, o);
      before += __shfl_xor_sync(0xffffffffu, before, o);
    }
    if (lane == 0) {
      keys[less + before] = key;
      places[less + before] = t;
      if (before == 0 && key < a.rows) ranges[key] = make_uint2(less, less + same);
    }
  }
}

// ------------------------------------------------------------------ gradient
constexpr u32 PIECE = 32, PIECE2 = PIECE * PIECE;
constexpr u32 LONG = 4096;     // from so many tokens on, pieces of 1024 are summed first (a launch; below, a list has up to 128 of 32)

struct GradientArgs {
  const u32 *keys, *places;    // sorted
  const uint2* ranges;
  float *sums, *sums2;         // of the pieces of 32 and of 1024 (or null), by the place of their first item / their size
  u32 n;
  u64 width;                   // of a row of sums: dim rounded up to whole packs
};

// N * LOADS sums of a lane, its columns 32 * N apart
template <int N, int LOADS>
struct Sum {
  float v[LOADS][N];
  __device__ __forceinline__ Sum() {
#pragma unroll
    for (int i = 0; i < LOADS; ++i)
#pragma unroll
      for (int e = 0; e < N; ++e) v[i][e] = 0.f;
  }
  // Adds `count` rows in order, AHEAD of them under way at once: row r is at base + place(r) * stride; `columns` of them
  // are left from this lane's first on.
  template <int AHEAD, class T, class Place>
  __device__ __forceinline__ void add_rows(const T* base, u64 stride, u32 count, s64 columns, Place place) {
#pragma unroll 1
    for (u32 r = 0; r < count; r += AHEAD) {
      Pack<T, N> p[AHEAD][LOADS];
#pragma unroll
      for (int q = 0; q < AHEAD; ++q) {
        const T* at = base + (u64)place(min(r + q, count - 1)) * stride;
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
          p[q][i].clear();
          if (r + q < count && i * 32 * N < columns) p[q][i].load(at + i * 32 * N);
        }
      }
#pragma unroll
      for (int q = 0; q < AHEAD; ++q)
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
          float x[N];
          p[q][i].widen(x);
#pragma unroll
          for (int e = 0; e < N; ++e) v[i][e] += x[e];
        }
    }
  }
};

// A piece of a list that begins among the items [size * w, size * w + size): its first item's place, or n.  Such a piece has the
// last of these items in it, so that there is one at most.
__device__ __forceinline__ u32 piece_in(const EmbedArgs& a, const GradientArgs& g, u32 w, u32 size) {
  const u32 last = w * size + size - 1;
  if (last >= g.n) return g.n;
  const u32 key = g.keys[last];
  if (key >= a.rows) return g.n;
  const uint2 range = g.ranges[key];
  const u32 first = last - (last - range.x) % size;
  return first + size <= range.y ? first : g.n;
}

// (A warp has few columns here, so that the pieces make many warps: a short list is a chain of loads.)
constexpr int PIECE_BLOCKS = 4, PIECE_BLOCKS_FEW = 1;
template <class T, int N, int AHEAD, int BLOCKS>
__global__ void __launch_bounds__(256, BLOCKS) k_pieces(EmbedArgs a, GradientArgs g, u32 chunks, Divider by_chunk, u32 items) {
  let_next_begin();
  wait_for_earlier();
  const u32 lane = threadIdx.x % 32, step = gridDim.x * 8;
  for (u32 item = blockIdx.x * 8 + threadIdx.x / 32; item < items; item += step) {
    const u32 w = by_chunk.of(item), first = piece_in(a, g, w, PIECE);
    if (first >= g.n) continue;
    const u64 column = (u64)(item - w * chunks) * (32 * N) + lane * N;
    const s64 columns = (s64)a.dim - (s64)column;
    const u32 place = g.places[first + lane];
    Sum<N, 1> sum;
    sum.template add_rows<AHEAD>((const T*)a.out + column, a.out_stride, PIECE, columns,
                             [&](u32 r) { return __shfl_sync(0xffffffffu, place, r); });
    if (columns > 0) {
      Pack<float, N> p;
      p.narrow(sum.v[0]);
      p.store(g.sums + w * g.width + column);
    }
  }
}

__global__ void __launch_bounds__(256, PIECE_BLOCKS) k_pieces2(EmbedArgs a, GradientArgs g, u32 chunks, Divider by_chunk, u32 items) {
  let_next_begin();
  wait_for_earlier();
  const u32 lane = threadIdx.x % 32, step = gridDim.x * 8;
  for (u32 item = blockIdx.x * 8 + threadIdx.x / 32; item < items; item += step) {
    const u32 w = by_chunk.of(item), first = piece_in(a, g, w, PIECE2);
    if (first >= g.n) continue;
    const u64 column = (u64)(item - w * chunks) * 128 + lane * 4;
    const s64 columns = (s64)g.width - (s64)column;       // (sums behind dim are there, and not used)
    Sum<4, 1> sum;
    sum.add_rows<8>(g.sums + column, g.width, PIECE, columns, [&](u32 r) { return first / PIECE + r; });
    if (columns > 0) {
      Pack<float, 4> p;
      p.narrow(sum.v[0]);
      p.store(g.sums2 + w * g.width + column);
    }
  }
}

// The gradient of one row, from `column` on (of which `columns` are left): its list is the places [at, end).
template <class T, class G, int N, int LOADS, int AHEAD>
__device__ __forceinline__ void write_row(const EmbedArgs& a, const GradientArgs& g, u32 at, u32 end, u64 column, s64 columns, G* to) {
  const u32 lane = threadIdx.x % 32, count = end - at;
  Sum<N, LOADS> sum;
  if (count >= PIECE) {
    if (g.sums2 && count >= PIECE2) {
      const u32 pieces = count / PIECE2;
      sum.template add_rows<2>(g.sums2 + column, g.width, pieces, columns, [&](u32 q) { return at / PIECE2 + q; });
      at += pieces * PIECE2;
    }
    const u32 pieces = (end - at) / PIECE;
    sum.template add_rows<2>(g.sums + column, g.width, pieces, columns, [&](u32 q) { return at / PIECE + q; });
    at += pieces * PIECE;
  }
  if (at < end) {
    const u32 place = at + lane < end ? g.places[at + lane] : 0;
    sum.template add_rows<AHEAD>((const T*)a.out + column, a.out_stride, end - at, columns,
                              [&](u32 q) { return __shfl_sync(0xffffffffu, place, q); });
  }
#pragma unroll
  for (int i = 0; i < LOADS; ++i)
    if (i * 32 * N < columns) {
      Pack<G, N> p;
      float x[N];
#pragma unroll
      for (int e = 0; e < N; ++e) x[e] = 0.f;
      if (a.accumulate) {
        p.load(to + i * 32 * N);
        p.widen(x);
      }
#pragma unroll
      for (int e = 0; e < N; ++e) x[e] = a.accumulate ? fmaf(sum.v[i][e], a.scale, x[e]) : sum.v[i][e] * a.scale;
      p.narrow(x);
      p.store(to + i * 32 * N);
    }
}

// A warp takes GROUP rows, LOADS packs a lane of each: their lists' bounds come in one load, so that rows without tokens, often
// most of them, are a store each and nothing is waited for.
template <class T, class G, int N, int GROUP, int LOADS, int AHEAD, int BLOCKS>
__global__ void __launch_bounds__(256, BLOCKS) k_gradient(EmbedArgs a, GradientArgs g, u32 chunks, Divider by_chunk, u32 items) {
  wait_for_earlier();
  const u32 lane = threadIdx.x % 32, step = gridDim.x * 8;
  auto ranges_of = [&](u32 item) {
    const u32 row = by_chunk.of(item) * GROUP + lane;
    return g.n && item < items && lane < GROUP && row < (u32)a.rows ? g.ranges[row] : make_uint2(0, 0);
  };
  u32 item = blockIdx.x * 8 + threadIdx.x / 32;
  uint2 next = ranges_of(item);
  for (; item < items; item += step) {
    const u32 first = by_chunk.of(item) * GROUP, rows = min((u32)GROUP, (u32)a.rows - first);
    const u64 column = (u64)(item - first / GROUP * chunks) * (32 * N * LOADS) + lane * N;
    const s64 columns = (s64)a.dim - (s64)column;
    const uint2 ranges = next;
    next = ranges_of(item + step);
    G* to = (G*)a.table + first * a.table_stride + column;
#pragma unroll 1
    for (u32 r = 0; r < rows; ++r, to += a.table_stride) {
      const u32 at = __shfl_sync(0xffffffffu, ranges.x, r), end = __shfl_sync(0xffffffffu, ranges.y, r);
      if (at == end) {
        if (!a.accumulate) {
          Pack<G, N> zero;
          zero.clear();
#pragma unroll
          for (int i = 0; i < LOADS; ++i)
            if (i * 32 * N < columns) zero.store(to + i * 32 * N);
        }
        continue;
      }
      write_row<T, G, N, LOADS, AHEAD>(a, g, at, end, column, columns, to);
    }
  }
}

// The rows that have tokens alone: a warp takes the place where a row's list begins, and leaves the others.
constexpr int LIST_BLOCKS = 5;
template <class T, class G, int N>
__global__ void __launch_bounds__(256, LIST_BLOCKS) k_lists(EmbedArgs a, GradientArgs g, u32 chunks, Divider by_chunk, u32 items) {
  wait_for_earlier();
  const u32 step = gridDim.x * 8;
  for (u32 item = blockIdx.x * 8 + threadIdx.x / 32; item < items; item += step) {
    const u32 place = by_chunk.of(item), key = g.keys[place];
    if (key >= a.rows || (place > 0 && g.keys[place - 1] == key)) continue;
    const u64 column = (u64)(item - place * chunks) * (32 * N) + threadIdx.x % 32 * N;
    write_row<T, G, N, 1, 4>(a, g, place, g.ranges[key].y, column, (s64)a.dim - (s64)column, (G*)a.table + key * a.table_stride + column);
  }
}

// ------------------------------------------------------------------ host
constexpr int FILL_BLOCKS = 8;
constexpr u64 SMALL_TABLE = (u64)1 << 25;
u32 chunks_of(u64 dim, int columns) { return (u32)((dim + columns - 1) / columns); }
// columns of a row of sums, for every size of packs
u64 width_of(u64 dim) { return (dim + 7) / 8 * 8; }

// How the radix sort goes: rows + 1 keys (the last one for tokens without a row), digits of up to 9 bits, a block for a
// tile of 2048 tokens, or for several where there would be more than 148 blocks: as many as the GPU has room for at once (each of them
// reads all blocks' counts).
constexpr u32 SORT_BLOCKS = 148;
SortArgs sort_plan(const EmbedArgs& a) {
  SortArgs s;
  memset(&s, 0, sizeof(s));
  s.n = (u32)a.n_tokens;
  u32 bits = 1;
  while (((u64)1 << bits) < a.rows + 1) ++bits;
  s.passes = (bits + MAX_BITS - 1) / MAX_BITS;
  s.bits = (bits + s.passes - 1) / s.passes;
  const u32 tiles = (s.n + SORT_TILE - 1) / SORT_TILE, a_block = tiles ? (tiles + SORT_BLOCKS - 1) / SORT_BLOCKS : 1;
  s.chunk = a_block * SORT_TILE;
  s.blocks = (s.n + s.chunk - 1) / s.chunk;
  return s;
}

struct Work {
  u32 *keys[2], *values[2], *counts;
  uint2* ranges;
  float *sums, *sums2;
  size_t bytes;
};
Work work_of(const EmbedArgs& a) {
  const SortArgs s = sort_plan(a);
  size_t at = 0;
  auto take = [&](size_t bytes) {
    char* p = (char*)a.work + at;
    at += (bytes + 255) / 256 * 256;
    return p;
  };
  Work w;
  for (int i = 0; i < 2; ++i) {
    w.keys[i] = (u32*)take(4 * (size_t)s.n);
    w.values[i] = (u32*)take(4 * (size_t)s.n);
  }
  w.counts = (u32*)take(s.n > RANK_MOST ? (size_t)s.blocks * 4 << s.bits : 0);
  w.ranges = (uint2*)take(8 * a.rows);
  w.sums = (float*)take(s.n / PIECE * width_of(a.dim) * 4);
  w.sums2 = (float*)take(s.n / PIECE2 * width_of(a.dim) * 4);
  w.bytes = a.n_tokens ? at : 0;
  return w;
}

// items of a grid: as many as a 31-bit index holds in one launch (each launch takes whole first coordinates)
template <class Launch>
cudaError_t in_parts(u64 count, u32 chunks, Launch launch) {
  const u64 most = 0x7fffffffu / chunks;
  for (u64 at = 0; at < count; at += most) {
    launch(at, (u32)(count - at < most ? count - at : most));
    const cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return e;
  }
  return cudaSuccess;
}
u32 grid_for(u32 items, int sm_count, int resident) {
  const u32 blocks = (items + 7) / 8, most = (u32)(sm_count * resident);
  return blocks < most ? blocks : most;
}

template <class T, int N>
cudaError_t lookup(const EmbedArgs& a, int sm_count, cudaStream_t stream) {
  const u32 chunks = chunks_of(a.dim, 32 * N * LOOKUP_LOADS<T, N>);
  return in_parts(a.n_tokens, chunks, [&](u64 at, u32 count) {
    EmbedArgs part = a;
    part.tokens = (const char*)a.tokens + at * a.token_bytes;
    part.out = (T*)a.out + at * a.out_stride;
    k_lookup<T, N><<<grid_for(count * chunks, sm_count, LOOKUP_BLOCKS), 256, 0, stream>>>(part, chunks, Divider(chunks), count * chunks);
  });
}

template <class T, class G, int N, int GROUP, int LOADS, int AHEAD, int BLOCKS>
cudaError_t write_rows(const EmbedArgs& a, const GradientArgs& g, int sm_count, cudaStream_t stream) {
  const u32 chunks = chunks_of(a.dim, 32 * N * LOADS);
  cudaError_t e = cudaSuccess;
  const cudaError_t e2 = in_parts((a.rows + GROUP - 1) / GROUP, chunks, [&](u64 at, u32 count) {
    EmbedArgs part = a;
    GradientArgs gp = g;
    part.table = (G*)a.table + at * GROUP * a.table_stride;
    part.rows = a.rows - at * GROUP;
    gp.ranges = g.ranges + (g.n ? at * GROUP : 0);
    const cudaError_t e1 = launch_next(k_gradient<T, G, N, GROUP, LOADS, AHEAD, BLOCKS>, grid_for(count * chunks, sm_count, BLOCKS), 256, 0,
                                       stream, part, gp, chunks, Divider(chunks), count * chunks);
    if (e1 != cudaSuccess) e = e1;
  });
  return e != cudaSuccess ? e : e2;
}

// The places and lists of few tokens, and zeros in the whole table
template <class G>
cudaError_t rank(const EmbedArgs& a, const Work& w, u32 n, int sm_count, cudaStream_t stream) {
  const u32 counting = grid_for(n, sm_count, 4), shared = (n + 3) / 4 * 16;
  const bool one = a.table_stride == a.dim, wide = aligned_rows(a.table, one ? a.rows * a.dim : a.table_stride, sizeof(G), 16) && (one || a.dim * sizeof(G) % 16 == 0);
  const u64 width = wide ? 16 : sizeof(G), bytes = (one ? a.rows * a.dim : a.dim) * sizeof(G);
  Fill f = {a.accumulate ? nullptr : (char*)a.table, bytes / width, a.table_stride * sizeof(G), one ? 1 : (u32)a.rows};
  const u64 parts = f.rows * ((f.units + 2047) / 2048), most = (u64)sm_count * FILL_BLOCKS;
  const u32 grid = counting + (f.table ? (u32)(parts < most ? parts : most) : 0);
  if (wide) k_rank<16><<<grid, 256, shared, stream>>>(a, n, w.keys[0], w.values[0], w.ranges, counting, f);
  else k_rank<sizeof(G)><<<grid, 256, shared, stream>>>(a, n, w.keys[0], w.values[0], w.ranges, counting, f);
  return cudaGetLastError();
}

template <class T, class G, int N>
cudaError_t gradient(const EmbedArgs& a, int sm_count, cudaStream_t stream) {
  cudaError_t e;
  GradientArgs g;
  memset((void*)&g, 0, sizeof(g));
  g.n = (u32)a.n_tokens;
  g.width = width_of(a.dim);
  const Work w = work_of(a);
  if (g.n) {
    SortArgs s = sort_plan(a);
    s.counts = w.counts;
    if (g.n <= RANK_MOST) {
      if ((e = rank<G>(a, w, g.n, sm_count, stream)) != cudaSuccess) return e;
    } else {
      if ((e = cudaMemsetAsync(w.ranges, 0, 8 * a.rows, stream)) != cudaSuccess) return e;
      for (u32 pass = 0; pass < s.passes; ++pass) {
        const int to = (s.passes - 1 - pass) & 1;
        s.shift = pass * s.bits;
        s.keys_in = pass ? w.keys[to ^ 1] : nullptr;
        s.values_in = pass ? w.values[to ^ 1] : nullptr;
        s.keys_out = w.keys[to];
        s.values_out = w.values[to];
        if (pass) e = launch_next(k_sort_count, s.blocks, SORT_THREADS, 0, stream, a, s);
        else k_sort_count<<<s.blocks, SORT_THREADS, 0, stream>>>(a, s), e = cudaGetLastError();
        if (e == cudaSuccess) e = launch_next(k_sort_place, s.blocks, SORT_THREADS, 0, stream, a, s);
        if (e != cudaSuccess) return e;
      }
      if ((e = launch_next(k_mark, (g.n + 255) / 256, 256, 0, stream, w.keys[0], g.n, w.ranges, a.rows)) != cudaSuccess) return e;
    }
    g.keys = w.keys[0];
    g.places = w.values[0];
    g.ranges = w.ranges;
    g.sums = w.sums;
    g.sums2 = g.n >= LONG ? w.sums2 : nullptr;
  }
  // (pieces number n / 32 at most, and a row of the sums is as long as d_out's: fewer items than 2^31 for any d_out that fits)
  if (g.n >= PIECE) {
    const u32 chunks = chunks_of(a.dim, 32 * N), items = g.n / PIECE * chunks;
    // pieces that all run at once are a chain of loads each: all of a piece's rows are loaded ahead
    if (items <= (u32)sm_count * 8 * PIECE_BLOCKS_FEW)
      e = launch_next(k_pieces<T, N, (int)PIECE, PIECE_BLOCKS_FEW>, (items + 7) / 8, 256, 0, stream, a, g, chunks, Divider(chunks), items);
    else
      e = launch_next(k_pieces<T, N, 8, PIECE_BLOCKS>, grid_for(items, sm_count, PIECE_BLOCKS), 256, 0, stream, a, g, chunks, Divider(chunks), items);
    if (e != cudaSuccess) return e;
  }
  if (g.n >= LONG) {
    const u32 chunks = chunks_of(g.width, 128), items = g.n / PIECE2 * chunks;
    if ((e = launch_next(k_pieces2, grid_for(items, sm_count, PIECE_BLOCKS), 256, 0, stream, a, g, chunks, Divider(chunks), items)) != cudaSuccess)
      return e;
  }
  if (g.n && g.n <= RANK_MOST) {
    const u32 chunks = chunks_of(a.dim, 32 * N);       // (up to 2^15, for up to 2^13 places)
    return launch_next(k_lists<T, G, N>, grid_for(g.n * chunks, sm_count, LIST_BLOCKS), 256, 0, stream, a, g, chunks, Divider(chunks), g.n * chunks);
  }
  // One pack a lane in small tables, two in large ones (bfloat16, L2 flushed before).  32768 tokens into 8000 x 512: 59 us with one, 66 with two;
  // 131072 into 256000 x 8192: 1188 and 1168.  Between 2^24 and 2^29 elements either is ahead, by 10 % at most (floats, 16000 x 1024: 104 and
  // 95; bfloat16, 32000 x 1152: 81 and 89; 64000 x 4096: 192 and 196; 128000 x 4096: 285 and 286).
  if (a.rows * a.dim <= SMALL_TABLE) return write_rows<T, G, N, 8, 1, 4, 5>(a, g, sm_count, stream);
  return write_rows<T, G, N, 8, 2, 4, 3>(a, g, sm_count, stream);
}

// packs of 16 bytes of the values that are read, where both tensors allow it
template <class T, class G>
cudaError_t gradient(const EmbedArgs& a, int sm_count, cudaStream_t stream) {
  constexpr int N = 16 / sizeof(T);
  if (a.dim % N == 0 && packs_at(a.out, a.out_stride, N, sizeof(T)) && packs_at(a.table, a.table_stride, N, sizeof(G)))
    return gradient<T, G, N>(a, sm_count, stream);
  return gradient<T, G, 1>(a, sm_count, stream);
}
template <class T>
cudaError_t gradient(u32 grad_dtype, const EmbedArgs& a, int sm_count, cudaStream_t stream) {
  if (grad_dtype == PS_F32) return gradient<T, float>(a, sm_count, stream);
  return grad_dtype == PS_BF16 ? gradient<T, __nv_bfloat16>(a, sm_count, stream) : gradient<T, __half>(a, sm_count, stream);
}
template <class T>
cudaError_t lookup(const EmbedArgs& a, int sm_count, cudaStream_t stream) {
  constexpr int N = 16 / sizeof(T);
  if (a.dim % (2 * N) == 0 && aligned_rows(a.out, a.out_stride, sizeof(T), 32) && aligned_rows(a.table, a.table_stride, sizeof(T), 32))
    return lookup<T, 2 * N>(a, sm_count, stream);
  if (a.dim % N == 0 && packs_at(a.out, a.out_stride, N, sizeof(T)) && packs_at(a.table, a.table_stride, N, sizeof(T)))
    return lookup<T, N>(a, sm_count, stream);
  return lookup<T, 1>(a, sm_count, stream);
}

}  // namespace

cudaError_t launch_embed_forward(u32 dtype, const EmbedArgs& a, int sm_count, cudaStream_t stream) {
  if (dtype == PS_F32) return lookup<float>(a, sm_count, stream);
  return dtype == PS_BF16 ? lookup<__nv_bfloat16>(a, sm_count, stream) : lookup<__half>(a, sm_count, stream);
}

size_t embed_backward_bytes(const EmbedArgs& a) { return work_of(a).bytes; }

cudaError_t launch_embed_backward(u32 dtype, u32 grad_dtype, const EmbedArgs& a, int sm_count, cudaStream_t stream) {
  if (dtype == PS_F32) return gradient<float>(grad_dtype, a, sm_count, stream);
  return dtype == PS_BF16 ? gradient<__nv_bfloat16>(grad_dtype, a, sm_count, stream) : gradient<__half>(grad_dtype, a, sm_count, stream);
}
