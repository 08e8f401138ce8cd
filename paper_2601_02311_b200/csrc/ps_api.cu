// The C interface: argument validation, host-side enumeration of the
// factorisations, scratch management and kernel launches.  No arithmetic of the
// method happens on the host; every evaluation runs in the kernels.
#include <cuda_runtime.h>
#include <math.h>
#include <stdlib.h>
#include <string.h>
#include <algorithm>
#include <atomic>
#include <chrono>
#include <cmath>
#include <initializer_list>
#include <new>
#include <vector>

#include "ps.h"
#include "ps_device.cuh"
#include "ps_internal.h"

namespace {

#define CUDA_OK(call)                         \
  do {                                        \
    if ((call) != cudaSuccess) return PS_E_CUDA; \
  } while (0)

struct DeviceGuard {
  int prev;
  bool ok;
  explicit DeviceGuard(int dev) : prev(-1), ok(false) {
    if (cudaGetDevice(&prev) != cudaSuccess) return;
    ok = (prev == dev) || cudaSetDevice(dev) == cudaSuccess;
  }
  ~DeviceGuard() {
    int cur = -1;
    if (prev >= 0 && cudaGetDevice(&cur) == cudaSuccess && cur != prev) cudaSetDevice(prev);
  }
};

bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }

// the supported ranges of a shape (the same limits the derivation kernel checks)
bool shape_in_range(const ps_model_shape& s, u32 tp_coll, u32 accum = 1) {
  if (s.layers < 1 || s.layers > (1u << 10)) return false;
  if (s.hidden < 1 || s.hidden > (1u << 16)) return false;
  if (s.heads < 1 || s.heads > (1u << 16)) return false;
  if (s.vocab < 1 || s.vocab > (1u << 24)) return false;
  if (s.seq < 1 || s.seq > (1u << 17)) return false;
  if (s.micro_batch < 1 || s.micro_batch > (1u << 10)) return false;
  const uint8_t w[4] = {s.w_param, s.w_grad, s.w_opt, s.w_act};
  for (int i = 0; i < 4; ++i)
    if (w[i] < 1 || w[i] > 16) return false;
  if (tp_coll > 64) return false;
  typedef unsigned __int128 u128;
  const u128 L = s.layers, H = s.hidden, V = s.vocab, S = s.seq, b = s.micro_batch, a = s.heads;
  const u128 P = s.param_elems_override ? (u128)s.param_elems_override : 12 * L * H * H + V * H;
  if (P < 1 || P > ((u128)1 << 46)) return false;
  if (S * b * H > ((u128)1 << 40)) return false;
  if (s.act_enabled) {
    const u128 A0 = L * (34 * S * b * H + 5 * a * S * S * b);
    if (A0 > ((u128)1 << 58)) return false;
    if (2 * A0 * accum > ((u128)1 << 62)) return false;        // host bytes of offloaded activations
  } else if (5 * a * S * S * b > ((u128)1 << 58)) {
    return false;
  }
  // tensor- and pipeline-axis bytes per step
  if ((L * 2 * tp_coll * s.w_act + 2 * s.w_act) * S * b * H * accum > ((u128)1 << 62)) return false;
  return true;
}

// whether every byte count of a (Theta, Omega, G) triple of this model -- device
// bytes (at most wsum * (P + 2 unit)), host bytes (at most (2 accum + 1) * wsum * P)
// and volume (data axis: at most (4 accum + 1) * wsum * P, with several copies of every
// shard 6 wsum * P more; tensor and pipeline axes as in shape_in_range) -- stays below 2^53
bool shape_is_small(const ps_model_shape& s, u32 tp_coll, u32 accum, u32 copies) {
  typedef unsigned __int128 u128;
  const u128 H = s.hidden;
  const u128 P = s.param_elems_override ? (u128)s.param_elems_override
                                        : 12 * (u128)s.layers * H * H + (u128)s.vocab * H;
  const u128 unit = s.unit_from_shape ? 12 * H * H : 0;
  const u128 wsum = (u128)s.w_param + s.w_grad + s.w_opt;
  const u128 axes = ((u128)s.layers * 2 * tp_coll * s.w_act + 2 * s.w_act) * s.seq * s.micro_batch * H * accum;
  return (4 * (u128)accum + 1 + (copies > 1 ? 6 : 0)) * wsum * (P + 2 * unit) + axes < ((u128)1 << 53);
}

int ensure_scratch(ps_ctx* ctx, size_t bytes) {
  if (bytes <= ctx->scratch_bytes) return PS_OK;
  CUDA_OK(cudaStreamSynchronize(ctx->stream));
  if (ctx->scratch) CUDA_OK(cudaFree(ctx->scratch));
  ctx->scratch = nullptr;
  ctx->scratch_bytes = 0;
  size_t want = (bytes + (size_t(1) << 20) - 1) & ~((size_t(1) << 20) - 1);
  CUDA_OK(cudaMalloc(&ctx->scratch, want));
  ctx->scratch_bytes = want;
  return PS_OK;
}

// ST_* bits of the problems that kernels have reported
u32 reported(const ps_ctx* ctx) {
  u32 st = 0;
  for (u32 b = 0; b < 8; ++b)
    if (ctx->h->status[b]) st |= 1u << b;
  return st;
}

// a problem that a kernel has reported by now
int pending_device_error(ps_ctx* ctx) {
  return reported(ctx) & ~(u32)ST_TRUNCATED ? PS_E_DEVICE : PS_OK;     // a truncated frontier blocks nothing
}

// Whether writing rows of `cols` elements at y (y_stride apart) may change what is still to be read of the
// rows at x: they share memory, and not as the very same elements, nor as column ranges of the same rows.
bool overwrites(const void* y, u64 y_stride, const void* x, u64 x_stride, u64 rows, u64 cols, u64 width) {
  if (y == x && (rows == 1 || y_stride == x_stride)) return false;
  const u64 ya = (u64)(uintptr_t)y, xa = (u64)(uintptr_t)x;
  const u64 y_end = ya + ((rows - 1) * y_stride + cols) * width, x_end = xa + ((rows - 1) * x_stride + cols) * width;
  if (y_end <= xa || x_end <= ya) return false;
  if (rows == 1 || y_stride != x_stride) return true;           // (a single row's strides say nothing, and may be 0)
  const u64 pitch = y_stride * width, off = (ya > xa ? ya - xa : xa - ya) % pitch;
  return off < cols * width || pitch - off < cols * width;
}

// What an operand takes of memory: `bytes` at all sums of up to three strides' multiples.  (bytes 0: nothing.)
typedef __int128 s128;
struct Region {
  static constexpr int DIMS = 3;
  s128 begin = 0, end = 0;
  u64 bytes = 0;
  u64 stride[DIMS] = {}, extent[DIMS] = {1, 1, 1};
  Region() {}
  Region(const void* p, u64 n, u64 width) : begin((uintptr_t)p), bytes(p ? n * width : 0) { close(); }
  Region(const ps_matrix& m, u64 rows, u64 cols, u64 width) : Region(rows ? m.data : nullptr, cols, width) { along(0, m.stride * width, rows); }
  Region(const ps_heads& h, u32 batch, u32 len, u32 heads, u64 dim, u64 width) : Region(h.data, dim, width) {
    along(0, h.batch_stride * width, batch), along(1, h.token_stride * width, len), along(2, h.head_stride * width, heads);
  }
  void along(int i, u64 by, u64 n) {
    if (n > 1 && by) stride[i] = by, extent[i] = n;
    close();
  }
  void close() {
    end = begin + bytes;
    for (int i = 0; i < DIMS; ++i) end += (s128)(extent[i] - 1) * stride[i];
  }
};
// Whether some whole numbers lo <= n <= hi, one for each stride, bring `apart` strictly between -below and above.  The longest strides come first, so that
// of each few numbers are left to try; where they are many after all, the answer is yes.
struct Reach {
  struct Term {
    s128 stride, lo, hi;
  };
  Term terms[2 * Region::DIMS];
  int count = 0, tries = 4096;
  void add(u64 stride, s128 lo, s128 hi) {
    int i = 0;
    while (i < count && terms[i].stride > stride) ++i;
    if (i < count && terms[i].stride == stride) {
      terms[i].lo += lo, terms[i].hi += hi;
      return;
    }
    for (int j = count++; j > i; --j) terms[j] = terms[j - 1];
    terms[i] = {stride, lo, hi};
  }
  bool within(s128 apart, s128 below, s128 above, int at = 0) {
    if (at == count) return -below < apart && apart < above;
    if (--tries < 0) return true;
    s128 low = 0, high = 0;                     // what the shorter strides can add
    for (int i = at + 1; i < count; ++i) low += terms[i].stride * terms[i].lo, high += terms[i].stride * terms[i].hi;
    const Term& t = terms[at];
    const auto floor = [&](s128 n) { return n >= 0 ? n / t.stride : -((-n + t.stride - 1) / t.stride); };
    const s128 first = std::max(t.lo, floor(-below - apart - high) + 1), last = std::min(t.hi, -floor(-(above - apart - low)) - 1);
    for (s128 n = first; n <= last; ++n)
      if (within(apart + n * t.stride, below, above, at + 1)) return true;
    return false;
  }
};
bool meet(const Region& a, const Region& b) {
  if (!a.bytes || !b.bytes || a.end <= b.begin || b.end <= a.begin) return false;
  Reach r;
  for (int i = 0; i < Region::DIMS; ++i) {
    if (a.extent[i] > 1) r.add(a.stride[i], 1 - (s128)a.extent[i], 0);
    if (b.extent[i] > 1) r.add(b.stride[i], 0, (s128)b.extent[i] - 1);
  }
  return r.within(b.begin - a.begin, b.bytes, a.bytes);
}
// whether a result meets one of these
bool meets(const Region& result, std::initializer_list<Region> others) {
  for (const Region& other : others)
    if (meet(result, other)) return true;
  return false;
}
// whether two of a result's own rows meet
bool meets_itself(const Region& a) {
  int order[Region::DIMS] = {0, 1, 2};
  std::sort(order, order + Region::DIMS, [&](int i, int j) { return a.stride[i] < a.stride[j]; });
  s128 reach = a.bytes;
  bool apart = true;                            // (as in most tensors: each stride is past all that the shorter ones reach)
  for (int i : order)
    if (a.extent[i] > 1) apart = apart && reach <= a.stride[i], reach += (s128)(a.extent[i] - 1) * a.stride[i];
  if (apart || a.bytes == 0) return false;
  for (int one = 0; one < Region::DIMS; ++one) {
    if (a.extent[one] == 1) continue;
    Reach r;
    for (int i = 0; i < Region::DIMS; ++i)
      if (a.extent[i] > 1) r.add(a.stride[i], i == one ? 1 : 1 - (s128)a.extent[i], (s128)a.extent[i] - 1);
    if (r.within(0, a.bytes, a.bytes)) return true;
  }
  return false;
}
bool same_rows(const ps_matrix& x, const ps_matrix& y, u64 rows) { return x.data == y.data && (rows == 1 || x.stride == y.stride); }

// flag bits a filter may require
constexpr u32 KNOWN_FLAGS = (PS_F_PAPER_PRICED << 1) - 1u;

}  // namespace

extern "C" {

const char* ps_strerror(int code) {
  switch (code) {
    case PS_OK: return "ok";
    case PS_E_NULLPTR: return "a required pointer is null";
    case PS_E_ALIGN: return "a device pointer is misaligned";
    case PS_E_RANGE: return "a size, shape or count is outside the supported range";
    case PS_E_BADINDEX: return "the index window leaves the space";
    case PS_E_TRUNCATED: return "an output was too short";
    case PS_E_CUDA: return "a CUDA runtime call failed";
    case PS_E_UNIMPLEMENTED: return "not implemented";
    case PS_E_DEVICE: return "a kernel reported an inconsistency";
    case PS_E_NOALLOC_LIMIT:
      return "the window needs more scratch than the no-allocation entry point's fixed array holds";
    default: return "unknown error";
  }
}

int ps_create(ps_ctx** out, int device, void* cuda_stream) {
  if (!out) return PS_E_NULLPTR;
  *out = nullptr;
  int n_dev = 0;
  if (cudaGetDeviceCount(&n_dev) != cudaSuccess || n_dev < 1) return PS_E_CUDA;
  if (device < 0 || device >= n_dev) return PS_E_RANGE;
  DeviceGuard guard(device);
  if (!guard.ok) return PS_E_CUDA;
  ps_ctx* ctx = new (std::nothrow) ps_ctx();
  if (!ctx) return PS_E_CUDA;
  ctx->device = device;
  ctx->stream = static_cast<cudaStream_t>(cuda_stream);
  ctx->scratch = nullptr;
  ctx->scratch_bytes = 0;
  ctx->d_lengths = nullptr;
  ctx->check = new (std::nothrow) std::mutex();
  ctx->h = nullptr;
  cudaDeviceProp prop;
  if (cudaGetDeviceProperties(&prop, device) != cudaSuccess) { ps_destroy(ctx); return PS_E_CUDA; }
  ctx->sm_count = prop.multiProcessorCount;
  if (!ctx->check || cudaMalloc(&ctx->d_lengths, 4 * sizeof(u32)) != cudaSuccess ||
      cudaHostAlloc(reinterpret_cast<void**>(&ctx->h), sizeof(HostWords), cudaHostAllocMapped | cudaHostAllocPortable) != cudaSuccess ||
      cudaMemsetAsync(ctx->d_lengths, 0, 4 * sizeof(u32), ctx->stream) != cudaSuccess) {
    ps_destroy(ctx);
    return PS_E_CUDA;
  }
  for (volatile u32& w : ctx->h->status) w = 0;
  ctx->h->answered = 0;
  ctx->checks = 0;
  if (ensure_scratch(ctx, size_t(8) << 20) != PS_OK) { ps_destroy(ctx); return PS_E_CUDA; }
  *out = ctx;
  return PS_OK;
}

void ps_destroy(ps_ctx* ctx) {
  if (!ctx) return;
  DeviceGuard guard(ctx->device);
  cudaStreamSynchronize(ctx->stream);
  if (ctx->scratch) cudaFree(ctx->scratch);
  if (ctx->d_lengths) cudaFree(ctx->d_lengths);
  if (ctx->h) cudaFreeHost(ctx->h);
  delete ctx->check;
  delete ctx;
}

int ps_status(ps_ctx* ctx) {
  if (!ctx) return PS_E_NULLPTR;
  DeviceGuard guard(ctx->device);
  if (!guard.ok) return PS_E_CUDA;
  CUDA_OK(cudaStreamSynchronize(ctx->stream));
  int rc = pending_device_error(ctx);
  if (rc == PS_OK && (reported(ctx) & ST_TRUNCATED)) rc = PS_E_TRUNCATED;
  if (rc != PS_OK)
    for (volatile u32& w : ctx->h->status) w = 0;
  return rc;
}

// The order in which the sweeps' blocks take the models: most expected work first, so
// that the blocks still running when the grid runs out are short ones.  A sweep block's
// duration grows with the number of factorisations that pass the composition tests for
// its model (T divides the heads, K divides the layers, T within the valid tensor
// degree): only those have survivors under a filter that requires a valid composition,
// and a unit with survivors costs several times one without.  The count is a sum over
// the distinct (T, K) pairs of the space, weighted by how many device counts have them.
static void sweep_degrees(ps_space* sp) {        // T -> (K, number of factorisations)
  auto& by_t = sp->degrees;
  for (const Fact& f : sp->facts) {
    if (f.T > sp->dev.tp_max_valid) continue;
    auto t = std::find_if(by_t.begin(), by_t.end(), [&](const auto& e) { return e.first == f.T; });
    if (t == by_t.end()) { by_t.push_back({f.T, {}}); t = by_t.end() - 1; }
    auto k = std::find_if(t->second.begin(), t->second.end(), [&](const auto& e) { return e.first == f.K; });
    if (k == t->second.end()) t->second.push_back({f.K, 1u}); else ++k->second;
  }
}
static void sweep_order(ps_space* sp, const ps_model_shape* models, u32 n_models) {
  std::vector<u32> work(n_models, 0);
  for (u32 i = 0; i < n_models; ++i)
    for (const auto& t : sp->degrees) {
      if (models[i].heads % t.first) continue;
      for (const auto& k : t.second)
        if (models[i].layers % k.first == 0) work[i] += k.second;
    }
  sp->order.resize(n_models);
  for (u32 i = 0; i < n_models; ++i) sp->order[i] = i;
  // (among models with the same count the smaller first: more of its points fit a capacity)
  std::stable_sort(sp->order.begin(), sp->order.end(), [&](u32 a, u32 b) {
    if (work[a] != work[b]) return work[a] > work[b];
    const u64 pa = (u64)models[a].layers * models[a].hidden * models[a].hidden;
    const u64 pb = (u64)models[b].layers * models[b].hidden * models[b].hidden;
    return pa < pb;
  });
}

// ------------------------------------------------------------------ space
int ps_space_create(ps_ctx* ctx, const ps_space_desc* desc, ps_space** out) {
  if (!ctx || !desc || !out || !desc->models || !desc->n_values) return PS_E_NULLPTR;
  *out = nullptr;
  if (desc->n_models < 1 || desc->n_models > (1u << 20)) return PS_E_RANGE;
  if (desc->n_n < 1 || desc->n_n > 64) return PS_E_RANGE;
  if (desc->t_enum_max < 1 || desc->k_enum_max < 1) return PS_E_RANGE;
  if (desc->n_act_variants < 1 || desc->n_act_variants > 2) return PS_E_RANGE;
  if (desc->n_tpa_variants < 1 || desc->n_tpa_variants > 2) return PS_E_RANGE;
  if ((desc->mode_mask & 0x1Fu) == 0 || (desc->mode_mask & ~0x1Fu)) return PS_E_RANGE;
  if (desc->tp_coll_per_layer > 64) return PS_E_RANGE;
  for (u32 i = 0; i < desc->n_n; ++i)
    if (desc->n_values[i] < 1 || desc->n_values[i] > (1u << 24)) return PS_E_RANGE;
  if (desc->sstar_units > 2 || desc->grad_accum_steps > 64 || desc->replication_k > (1u << 24)) return PS_E_RANGE;
  const u32 accum = desc->grad_accum_steps ? desc->grad_accum_steps : 1;
  for (u32 i = 0; i < desc->n_models; ++i)
    if (!shape_in_range(desc->models[i], desc->tp_coll_per_layer, accum)) return PS_E_RANGE;

  DeviceGuard guard(ctx->device);
  if (!guard.ok) return PS_E_CUDA;
  ps_space* sp = new (std::nothrow) ps_space();
  if (!sp) return PS_E_CUDA;
  sp->ctx = ctx;
  sp->desc = *desc;
  sp->desc.models = nullptr;
  sp->desc.n_values = nullptr;
  sp->d_shapes = nullptr;
  sp->d_recs = nullptr;
  sp->d_facts = nullptr;
  sp->d_order = nullptr;
  sp->n_values.assign(desc->n_values, desc->n_values + desc->n_n);
  // all (T, K) with T | N, K | N/T inside the enumeration limits: T ascending, then K
  for (u32 i = 0; i < desc->n_n; ++i) {
    sp->fact_begin.push_back((u32)sp->facts.size());
    const u32 N = desc->n_values[i];
    std::vector<u32> sorted;                      // divisors of N, ascending
    for (u32 d = 1; (u64)d * d <= N; ++d)
      if (N % d == 0) { sorted.push_back(d); if (d != N / d) sorted.push_back(N / d); }
    std::sort(sorted.begin(), sorted.end());
    for (u32 T : sorted) {
      if (T > desc->t_enum_max) break;
      const u32 rest = N / T;
      for (u32 K : sorted) {
        if (K > desc->k_enum_max || K > rest) break;
        if (rest % K) continue;
        sp->facts.push_back(Fact{N, T, K, rest / K});
      }
    }
    if (sp->facts.size() > (size_t(1) << 20)) { delete sp; return PS_E_RANGE; }
  }
  sp->fact_begin.push_back((u32)sp->facts.size());
  if (sp->facts.empty()) { delete sp; return PS_E_RANGE; }
  u32 modemap = 0, nm = 0;
  for (u32 m = 0; m < 5; ++m)
    if (desc->mode_mask & (1u << m)) { modemap |= m << (4 * nm); sp->modes.push_back(m); ++nm; }
  SpaceDev& d = sp->dev;
  d.n_models = desc->n_models;
  d.n_facts = (u32)sp->facts.size();
  d.nv = desc->n_act_variants;
  d.nt = desc->n_tpa_variants;
  d.nvt = d.nv * d.nt;
  d.nm = nm;
  d.modemap = modemap;
  d.n3 = nm * nm * nm;
  d.n_codes = d.n3 * nm;
  d.tp_max_valid = desc->tp_max_valid;
  d.tp_coll = desc->tp_coll_per_layer;
  d.sstar_units = desc->sstar_units ? desc->sstar_units : 1;
  d.accum = accum;
  d.repl = desc->replication_k ? desc->replication_k : 1;
  d.all_pow2 = 1;
  for (u32 i = 0; i < desc->n_n; ++i)
    if (desc->n_values[i] & (desc->n_values[i] - 1)) d.all_pow2 = 0;
  const u64 ppm = (u64)d.n_facts * d.nvt * d.n_codes;
  if (ppm >= ((u64)1 << 32)) { delete sp; return PS_E_RANGE; }
  d.ppm = ppm;

  bool ok = cudaMalloc(&sp->d_shapes, sizeof(ps_model_shape) * (size_t)desc->n_models) == cudaSuccess &&
            cudaMalloc(&sp->d_recs, sizeof(ModelRec) * (size_t)desc->n_models) == cudaSuccess &&
            cudaMalloc(&sp->d_facts, sizeof(Fact) * sp->facts.size()) == cudaSuccess &&
            cudaMalloc(&sp->d_order, sizeof(u32) * (size_t)desc->n_models) == cudaSuccess;
  ok = ok && cudaMemcpyAsync(sp->d_facts, sp->facts.data(), sizeof(Fact) * sp->facts.size(),
                             cudaMemcpyHostToDevice, ctx->stream) == cudaSuccess;
  if (!ok) { ps_space_destroy(sp); return PS_E_CUDA; }
  d.recs = sp->d_recs;
  d.facts = sp->d_facts;
  d.order = sp->d_order;
  sweep_degrees(sp);
  int rc = ps_space_set_models(sp, desc->models, desc->n_models);
  if (rc == PS_OK && cudaStreamSynchronize(ctx->stream) != cudaSuccess) rc = PS_E_CUDA;
  if (rc != PS_OK) { ps_space_destroy(sp); return rc; }
  *out = sp;
  return PS_OK;
}

int ps_space_set_models(ps_space* sp, const ps_model_shape* models, uint32_t n_models) {
  if (!sp || !models) return PS_E_NULLPTR;
  if (n_models != sp->dev.n_models) return PS_E_RANGE;
  u32 all_small = 1;
  for (u32 i = 0; i < n_models; ++i) {
    if (!shape_in_range(models[i], sp->dev.tp_coll, sp->dev.accum)) return PS_E_RANGE;
    if (!shape_is_small(models[i], sp->dev.tp_coll, sp->dev.accum, sp->dev.repl)) all_small = 0;
  }
  sp->dev.all_small = all_small;
  ps_ctx* ctx = sp->ctx;
  DeviceGuard guard(ctx->device);
  if (!guard.ok) return PS_E_CUDA;
  // (blocks of a table that fits the GPU at once all start together: any order will do,
  // and the one that is there stays)
  const bool by_work = n_models > (u32)ctx->sm_count;
  if (by_work || sp->order.empty()) {
    if (by_work) {
      sweep_order(sp, models, n_models);
    } else {
      sp->order.resize(n_models);
      for (u32 i = 0; i < n_models; ++i) sp->order[i] = i;
    }
    CUDA_OK(cudaMemcpyAsync(sp->d_order, sp->order.data(), sizeof(u32) * (size_t)n_models, cudaMemcpyHostToDevice,
                            ctx->stream));
  }
  CUDA_OK(cudaMemcpyAsync(sp->d_shapes, models, sizeof(ps_model_shape) * (size_t)n_models,
                          cudaMemcpyHostToDevice, ctx->stream));
  CUDA_OK(launch_model_derive(sp->d_shapes, sp->d_recs, n_models, ctx->h->status, ctx->stream));
  return PS_OK;
}

int ps_space_rederive(ps_space* sp) {
  if (!sp) return PS_E_NULLPTR;
  ps_ctx* ctx = sp->ctx;
  DeviceGuard guard(ctx->device);
  if (!guard.ok) return PS_E_CUDA;
  CUDA_OK(launch_model_derive(sp->d_shapes, sp->d_recs, sp->dev.n_models, ctx->h->status, ctx->stream));
  return PS_OK;
}

void ps_space_destroy(ps_space* sp) {
  if (!sp) return;
  DeviceGuard guard(sp->ctx->device);
  cudaStreamSynchronize(sp->ctx->stream);
  if (sp->d_shapes) cudaFree(sp->d_shapes);
  if (sp->d_recs) cudaFree(sp->d_recs);
  if (sp->d_facts) cudaFree(sp->d_facts);
  if (sp->d_order) cudaFree(sp->d_order);
  delete sp;
}

uint64_t ps_space_size(const ps_space* sp) { return sp ? sp->dev.ppm * sp->dev.n_models : 0; }
uint64_t ps_space_points_per_model(const ps_space* sp) { return sp ? sp->dev.ppm : 0; }

int ps_space_decode(const ps_space* sp, uint64_t idx, ps_point* out) {
  if (!sp || !out) return PS_E_NULLPTR;
  if (idx >= ps_space_size(sp)) return PS_E_BADINDEX;
  const SpaceDev& d = sp->dev;
  out->model = (u32)(idx / d.ppm);
  u64 r = idx % d.ppm;
  const u64 per_unit = (u64)d.nvt * d.n_codes;
  const Fact& f = sp->facts[(size_t)(r / per_unit)];
  r %= per_unit;
  out->N = f.N; out->T = f.T; out->K = f.K; out->D = f.D;
  const u32 vt = (u32)(r / d.n_codes);
  u32 code = (u32)(r % d.n_codes);
  out->act_variant = vt / d.nt;
  out->tpa_variant = vt % d.nt;
  u32 full = 0, weight = 1;
  for (int s = 0; s < 4; ++s) {
    full += weight * sp->modes[code % d.nm];
    code /= d.nm;
    weight *= 5;
  }
  out->code_dp = (uint16_t)full;
  out->code_tp = out->tpa_variant == 0 ? PS_CODE_TP_SEQPAR : PS_CODE_TP;
  out->code_pp = PS_CODE_PP;
  out->pad = 0;
  return PS_OK;
}

// ------------------------------------------------------------------ batch evaluation
int ps_eval_batch(ps_ctx* ctx, const ps_space* sp, uint64_t first, uint64_t count,
                  const ps_filter* filter, ps_out_soa out, uint64_t* d_idx_out, uint64_t* d_n_out) {
  if (!ctx || !sp) return PS_E_NULLPTR;
  if (sp->ctx != ctx) return PS_E_RANGE;
  const u64 size = ps_space_size(sp);
  if (first > size || count > size - first) return PS_E_BADINDEX;
  if (filter && !d_n_out) return PS_E_NULLPTR;
  if (!aligned(out.mem, 8) || !aligned(out.comm_paper, 8) || !aligned(out.comm_ext, 8) ||
      !aligned(out.host, 8) || !aligned(out.flags, 4) || !aligned(d_idx_out, 8) || !aligned(d_n_out, 8))
    return PS_E_ALIGN;
  if (filter && (filter->comm_kind > PS_COMM_PAPER_PLUS_EXT || (filter->require_flags & ~KNOWN_FLAGS)))
    return PS_E_RANGE;
  int rc = pending_device_error(ctx);
  if (rc != PS_OK) return rc;
  DeviceGuard guard(ctx->device);
  if (!guard.ok) return PS_E_CUDA;
  if (count == 0) {
    if (filter) CUDA_OK(cudaMemsetAsync(d_n_out, 0, sizeof(u64), ctx->stream));
    return PS_OK;
  }
  EvalArgs a;
  memset(&a, 0, sizeof(a));
  a.first = first;
  a.count = count;
  a.first_group = first / sp->dev.n_codes;
  const u64 last_group = (first + count - 1) / sp->dev.n_codes;
  const u64 n_groups = last_group - a.first_group + 1;
  if (n_groups > (u64)0x7fffffff) return PS_E_RANGE;
  a.n_tiles = (u32)n_groups;
  a.out = out;
  a.idx_out = d_idx_out;
  a.n_out = d_n_out;
  if (!filter) {
    CUDA_OK(launch_eval_materialise(sp->dev, a, ctx->stream));
  } else {
    a.cap_bytes = filter->cap_bytes;
    a.host_cap = filter->host_cap;
    a.require_flags = filter->require_flags & ~(u32)PS_F_FEASIBLE;
    // per group an offset and a place in the list of factorisations with survivors, per run of
    // factorisations an offset
    eval_plan_runs(sp->dev, a);
    const size_t group_bytes = (sizeof(u32) * n_groups + 15) & ~size_t(15);
    rc = ensure_scratch(ctx, 2 * group_bytes + sizeof(u64) * (size_t)a.n_runs);
    if (rc != PS_OK) return rc;
    char* base = static_cast<char*>(ctx->scratch);
    a.group_offset = reinterpret_cast<u32*>(base);
    a.nonempty = reinterpret_cast<u32*>(base + group_bytes);
    a.run_offset = reinterpret_cast<u64*>(base + 2 * group_bytes);
    a.n_nonempty = ctx->d_lengths;
    a.n_listed = ctx->d_lengths + 1;
    a.blocks_done = ctx->d_lengths + 2;
    CUDA_OK(launch_eval_count(sp->dev, a, ctx->stream));
    CUDA_OK(launch_eval_write(sp->dev, a, ctx->stream));
  }
  return PS_OK;
}

// ------------------------------------------------------------------ sweeps
int ps_sweep_pareto(ps_ctx* ctx, const ps_space* sp, const ps_filter* filter,
                    const uint64_t* caps_bytes, uint32_t n_caps, uint32_t reduce_kind,
                    uint32_t max_entries, ps_front_entry* d_out, uint32_t* d_counts) {
  if (!ctx || !sp || !filter || !caps_bytes || !d_out || !d_counts) return PS_E_NULLPTR;
  if (sp->ctx != ctx) return PS_E_RANGE;
  if (n_caps < 1 || n_caps > PS_MAX_CAPS || max_entries < 1) return PS_E_RANGE;
  if (reduce_kind != PS_REDUCE_PARETO && reduce_kind != PS_REDUCE_TOPK) return PS_E_RANGE;
  if (reduce_kind == PS_REDUCE_TOPK && max_entries > PS_TOPK_MAX) return PS_E_RANGE;
  if (filter->comm_kind > PS_COMM_PAPER_PLUS_EXT || (filter->require_flags & ~KNOWN_FLAGS)) return PS_E_RANGE;
  if (!aligned(d_out, 8) || !aligned(d_counts, 4)) return PS_E_ALIGN;
  int rc = pending_device_error(ctx);
  if (rc != PS_OK) return rc;
  DeviceGuard guard(ctx->device);
  if (!guard.ok) return PS_E_CUDA;

  SweepArgs s;
  memset(&s, 0, sizeof(s));
  for (u32 c = 0; c < n_caps; ++c) {
    s.caps[c] = caps_bytes[c];
    s.cap_max = std::max(s.cap_max, s.caps[c]);
  }
  s.host_cap = filter->host_cap;
  s.require_flags = filter->require_flags & ~(u32)PS_F_FEASIBLE;
  s.comm_kind = filter->comm_kind;
  s.n_caps = n_caps;
  s.max_entries = max_entries;
  s.skip_rejected = filter->skip_rejected ? 1u : 0u;
  s.out = d_out;
  s.counts = d_counts;
  s.status = ctx->h->status;
  CUDA_OK(launch_sweep((int)reduce_kind, sp->dev, s, ctx->sm_count, ctx->stream));
  return PS_OK;
}

// ------------------------------------------------------------------ one composition
int ps_check_composition(ps_ctx* ctx, const ps_model_shape* shape, uint32_t N, uint32_t T,
                         uint32_t K, uint32_t D, uint16_t code_tp, uint16_t code_pp,
                         uint16_t code_dp, uint32_t act_variant, uint64_t cap_bytes,
                         uint32_t tp_max_valid, uint32_t tp_coll_per_layer, uint32_t comm_kind,
                         ps_front_entry* h_out) {
  if (!ctx || !shape || !h_out) return PS_E_NULLPTR;
  if (N < 1 || N > (1u << 24) || T < 1 || T > (1u << 24) || K < 1 || K > (1u << 24) || D < 1 ||
      D > (1u << 24))
    return PS_E_RANGE;
  if (code_tp > 624 || code_pp > 624 || code_dp > 624 || act_variant > 1 ||
      comm_kind > PS_COMM_PAPER_PLUS_EXT)
    return PS_E_RANGE;
  if (!shape_in_range(*shape, tp_coll_per_layer)) return PS_E_RANGE;
  DeviceGuard guard(ctx->device);
  if (!guard.ok) return PS_E_CUDA;
  // Table 2: tensor axis (S,S,S,S) or (S,S,S,R), pipeline axis (S,S,S,R); an axis
  // of degree 1 is absent.  Activation mode of the tensor axis: digit 3 of its code.
  const bool tp_form = (T == 1) || code_tp == PS_CODE_TP_SEQPAR || code_tp == PS_CODE_TP;
  const bool pp_form = (K == 1) || code_pp == PS_CODE_PP;
  const u32 tau = ((code_tp / 125) % 5 == PS_MODE_S) ? 0 : 1;
  // The shape travels with the launch and the answer comes back through mapped memory.  Its
  // arrival is looked for directly for a millisecond at most (longer if other work is before
  // it in the stream): waiting for the stream instead takes 5 us longer.
  std::lock_guard<std::mutex> lock(*ctx->check);
  const u32 call = ++ctx->checks;
  CUDA_OK(launch_check_point(*shape, Fact{N, T, K, D}, act_variant, tau, code_dp, tp_max_valid,
                             tp_coll_per_layer, (tp_form && pp_form) ? 1 : 0, comm_kind, cap_bytes,
                             ctx->h, call, ctx->stream));
  const auto begin = std::chrono::steady_clock::now();
  bool there = false;
  for (u32 k = 1; !(there = ctx->h->answered == call); ++k)
    if (k % 64 == 0 && std::chrono::steady_clock::now() - begin > std::chrono::milliseconds(1)) break;
  if (!there) CUDA_OK(cudaStreamSynchronize(ctx->stream));
  std::atomic_thread_fence(std::memory_order_acquire);
  *h_out = ctx->h->entry;
  return PS_OK;
}

// ------------------------------------------------------------------ Algorithm 1
int ps_select(ps_ctx* ctx, const ps_select_query* d_queries, uint64_t n, uint32_t headroom_num,
              uint32_t headroom_den, uint32_t layer_num, uint32_t layer_den, uint32_t tp_degree,
              ps_select_result* d_out) {
  if (!ctx || (n && (!d_queries || !d_out))) return PS_E_NULLPTR;
  if (!aligned(d_queries, 16) || !aligned(d_out, 16)) return PS_E_ALIGN;
  if (headroom_den < 1 || layer_den < 1 || tp_degree < 1 || headroom_num > (1u << 16) ||
      headroom_den > (1u << 16) || layer_num > (1u << 16) || layer_den > (1u << 16) ||
      n > ((u64)1 << 38))
    return PS_E_RANGE;
  if (n == 0) return PS_OK;
  DeviceGuard guard(ctx->device);
  if (!guard.ok) return PS_E_CUDA;
  CUDA_OK(launch_select(d_queries, n, headroom_num, headroom_den, layer_num, layer_den, tp_degree, d_out,
                        ctx->stream));
  return PS_OK;
}

int ps_select_compare(ps_ctx* ctx, const ps_space* sp, uint32_t n_index, uint64_t device_bytes,
                      uint32_t fast_interconnect, uint32_t headroom_num, uint32_t headroom_den,
                      uint32_t layer_num, uint32_t layer_den, uint32_t tp_degree, const ps_filter* filter,
                      const ps_front_entry* d_frontier, const uint32_t* d_counts, uint32_t n_caps,
                      uint32_t cap_index, uint32_t max_entries, ps_select_compare_result* d_out) {
  if (!ctx || !sp || !filter || !d_frontier || !d_counts || !d_out) return PS_E_NULLPTR;
  if (sp->ctx != ctx) return PS_E_RANGE;
  if (!aligned(d_frontier, 8) || !aligned(d_counts, 4) || !aligned(d_out, 8)) return PS_E_ALIGN;
  if (n_index >= sp->n_values.size() || n_caps < 1 || n_caps > PS_MAX_CAPS || cap_index >= n_caps || max_entries < 1 ||
      headroom_den < 1 || layer_den < 1 || tp_degree < 1 || headroom_num > (1u << 16) || headroom_den > (1u << 16) ||
      layer_num > (1u << 16) || layer_den > (1u << 16) || device_bytes > ((u64)1 << 50) ||
      filter->comm_kind > PS_COMM_PAPER_PLUS_EXT || (filter->require_flags & ~KNOWN_FLAGS))
    return PS_E_RANGE;
  int rc = pending_device_error(ctx);
  if (rc != PS_OK) return rc;
  DeviceGuard guard(ctx->device);
  if (!guard.ok) return PS_E_CUDA;
  CUDA_OK(launch_select_compare(sp->dev, sp->fact_begin[n_index], sp->fact_begin[n_index + 1], sp->n_values[n_index],
                                device_bytes, fast_interconnect, headroom_num, headroom_den, layer_num, layer_den,
                                tp_degree, filter->host_cap, filter->require_flags & ~(u32)PS_F_FEASIBLE,
                                filter->comm_kind, d_frontier, d_counts, n_caps, cap_index, max_entries, d_out,
                                ctx->stream));
  return PS_OK;
}

// ------------------------------------------------------------------ verification protocol
int ps_verify_batch(ps_ctx* ctx, const ps_verify_shape* shape, const ps_verify_case* d_cases, uint64_t n,
                    const double* d_data, uint64_t data_len, ps_verify_result* d_out, double* d_theta_out) {
  if (!ctx || !shape || (n && (!d_cases || !d_data || !d_out))) return PS_E_NULLPTR;
  if (!aligned(d_cases, 8) || !aligned(d_data, 8) || !aligned(d_out, 8) || !aligned(d_theta_out, 8)) return PS_E_ALIGN;
  const ps_verify_shape& s = *shape;
  if (s.units < 1 || s.units > 8 || s.h < 1 || s.h > 32 || s.b < 1 || s.b > 4 || s.accum < 1 || s.accum > 4 ||
      s.steps < 1 || s.steps > 16 || s.gather_buffers < 1 || s.gather_buffers > 2)
    return PS_E_RANGE;
  if (s.w_theta < 1 || s.w_theta > 16 || s.w_grad < 1 || s.w_grad > 16 || s.w_omega < 3 || s.w_omega > 48 ||
      s.w_omega % 3 != 0)
    return PS_E_RANGE;
  if (!(s.lr > 0) || !(s.beta1 >= 0 && s.beta1 < 1) || !(s.beta2 >= 0 && s.beta2 < 1) || !(s.eps > 0) ||
      !(s.rtol >= 0) || !(s.atol >= 0) || n > ((u64)1 << 32))
    return PS_E_RANGE;
  int rc = pending_device_error(ctx);
  if (rc != PS_OK) return rc;
  if (n == 0) return PS_OK;
  DeviceGuard guard(ctx->device);
  if (!guard.ok) return PS_E_CUDA;
  CUDA_OK(launch_verify(s, d_cases, n, d_data, data_len, d_theta_out, d_out, ctx->h->status, ctx->stream));
  return PS_OK;
}

// ------------------------------------------------------------ operators of a training step
int ps_dropout(ps_ctx* ctx, const ps_dropout_desc* desc, const void* d_x, const void* d_residual, void* d_y) {
  if (!ctx || !desc) return PS_E_NULLPTR;
  const ps_dropout_desc& d = *desc;
  if (d.dtype > PS_F16 || !(d.p >= 0 && d.p <= 1)) return PS_E_RANGE;
  if (d.rows == 0 || d.cols == 0) return PS_OK;
  if (!d_x || !d_y) return PS_E_NULLPTR;
  const u64 width = d.dtype == PS_F32 ? 4 : 2;
  if (!aligned(d_x, width) || !aligned(d_residual, width) || !aligned(d_y, width)) return PS_E_ALIGN;
  typedef unsigned __int128 u128;
  const u64 stride_most = (u64)1 << 40;
  if ((u128)d.rows * d.cols > (u128)1 << 48 || (d.rows > 1 && d.cols > ((u64)1 << 32)) || d.x_stride > stride_most || d.residual_stride > stride_most ||
      d.y_stride > stride_most || (d.rows > 1 && d.y_stride < d.cols) ||
      (u128)d.first + (u128)d.rows * d.pitch + d.cols > (u128)1 << 63)
    return PS_E_RANGE;
  if (overwrites(d_y, d.y_stride, d_x, d.x_stride, d.rows, d.cols, width) ||
      (d_residual && overwrites(d_y, d.y_stride, d_residual, d.residual_stride, d.rows, d.cols, width)))
    return PS_E_RANGE;
  int rc = pending_device_error(ctx);
  if (rc != PS_OK) return rc;
  DeviceGuard guard(ctx->device);
  if (!guard.ok) return PS_E_CUDA;
  DropoutArgs a;
  memset(&a, 0, sizeof(a));
  a.x = d_x; a.residual = d_residual; a.y = d_y;
  a.rows = d.rows; a.cols = d.cols;
  a.x_stride = d.x_stride; a.residual_stride = d.residual_stride; a.y_stride = d.y_stride;
  a.first = d.first; a.pitch = d.pitch; a.seed = d.seed; a.stream = d.stream;
  a.threshold = (u64)rint(d.p * 4294967296.0);
  a.scale = d.p < 1 ? (float)(1.0 / (1.0 - d.p)) : 0.f;
  CUDA_OK(launch_dropout(d.dtype, a, ctx->sm_count, ctx->stream));
  return PS_OK;
}

static int embed_args(const ps_embed_desc& d, EmbedArgs& a) {
  if (d.tokens > ((u64)1 << 30) || d.rows < 1 || d.rows > ((u64)1 << 30) || d.dim < 1 || d.dim > ((u64)1 << 20) ||
      d.table_stride < d.dim || d.out_stride < d.dim || d.table_stride > ((u64)1 << 32) || d.out_stride > ((u64)1 << 32) ||
      d.dtype > PS_F16 || d.grad_dtype > PS_F16 || (d.token_bytes != 4 && d.token_bytes != 8) || d.accumulate > 1 ||
      !std::isfinite((float)d.scale))
    return PS_E_RANGE;
  memset(&a, 0, sizeof(a));
  a.n_tokens = d.tokens; a.first_row = d.first_row; a.rows = d.rows; a.dim = d.dim;
  a.table_stride = d.table_stride; a.out_stride = d.out_stride;
  a.scale = (float)d.scale;
  a.token_bytes = d.token_bytes; a.accumulate = d.accumulate;
  return PS_OK;
}

int ps_embed_forward(ps_ctx* ctx, const ps_embed_desc* desc, const void* d_table, const void* d_tokens, void* d_out) {
  if (!ctx || !desc) return PS_E_NULLPTR;
  EmbedArgs a;
  int rc = embed_args(*desc, a);
  if (rc != PS_OK) return rc;
  if (a.n_tokens == 0) return PS_OK;
  if (!d_table || !d_tokens || !d_out) return PS_E_NULLPTR;
  const size_t width = desc->dtype == PS_F32 ? 4 : 2;
  if (!aligned(d_table, width) || !aligned(d_out, width) || !aligned(d_tokens, a.token_bytes)) return PS_E_ALIGN;
  if ((rc = pending_device_error(ctx)) != PS_OK) return rc;
  DeviceGuard guard(ctx->device);
  if (!guard.ok) return PS_E_CUDA;
  a.table = const_cast<void*>(d_table); a.tokens = d_tokens; a.out = d_out;
  CUDA_OK(launch_embed_forward(desc->dtype, a, ctx->sm_count, ctx->stream));
  return PS_OK;
}

uint64_t ps_embed_backward_bytes(const ps_embed_desc* desc) {
  EmbedArgs a;
  return desc && embed_args(*desc, a) == PS_OK ? embed_backward_bytes(a) : 0;
}

int ps_embed_backward(ps_ctx* ctx, const ps_embed_desc* desc, const void* d_out_grad, const void* d_tokens,
                      void* d_table_grad, void* d_work, uint64_t work_bytes) {
  if (!ctx || !desc || !d_table_grad) return PS_E_NULLPTR;
  EmbedArgs a;
  int rc = embed_args(*desc, a);
  if (rc != PS_OK) return rc;
  const u64 need = embed_backward_bytes(a);
  if ((a.n_tokens && (!d_out_grad || !d_tokens)) || (need && !d_work)) return PS_E_NULLPTR;
  if (!aligned(d_out_grad, desc->dtype == PS_F32 ? 4 : 2) || !aligned(d_table_grad, desc->grad_dtype == PS_F32 ? 4 : 2) ||
      !aligned(d_tokens, a.token_bytes) || !aligned(d_work, 256))
    return PS_E_ALIGN;
  if (work_bytes < need) return PS_E_RANGE;
  if ((rc = pending_device_error(ctx)) != PS_OK) return rc;
  DeviceGuard guard(ctx->device);
  if (!guard.ok) return PS_E_CUDA;
  a.table = d_table_grad; a.tokens = d_tokens; a.out = const_cast<void*>(d_out_grad); a.work = d_work;
  CUDA_OK(launch_embed_backward(desc->dtype, desc->grad_dtype, a, ctx->sm_count, ctx->stream));
  return PS_OK;
}

static int attention_args(const ps_attention_shape& s, AttentionArgs& a) {
  if (s.batch > 65535 || s.q_len > (1u << 24) || s.k_len > (1u << 24) || s.heads < 1 || s.heads > 32768 || s.kv_heads < 1 ||
      s.heads % s.kv_heads || s.dim < 8 || s.dim > 128 || s.dim % 8 || (s.dtype != PS_BF16 && s.dtype != PS_F16) ||
      s.causal > 1 || !std::isfinite(s.scale))
    return PS_E_RANGE;
  // what the grids can hold (a block for 128 queries or keys of a head in one dimension; rows by 8 or more, heads and sequences in three)
  if ((u64)s.batch * s.heads * ((std::max(s.q_len, s.k_len) + 127) / 128) > (1u << 26)) return PS_E_RANGE;
  memset(&a, 0, sizeof(a));
  a.batch = (int)s.batch; a.q_len = (int)s.q_len; a.k_len = (int)s.k_len;
  a.heads = (int)s.heads; a.kv_heads = (int)s.kv_heads; a.dim = (int)s.dim; a.causal = (int)s.causal;
  a.scale = s.scale;
  return PS_OK;
}

// a tensor [batch][len][heads][dim] of attention, and what has to hold of it
static int take_heads(const ps_heads* h, u32 batch, u32 len, u32 heads, ps_heads& into) {
  if (!h) return PS_E_NULLPTR;
  into = *h;
  if (batch == 0 || len == 0) return PS_OK;                     // no element is touched
  if (!h->data) return PS_E_NULLPTR;
  if (!aligned(h->data, 16)) return PS_E_ALIGN;
  u64* strides[3] = {&into.batch_stride, &into.token_stride, &into.head_stride};
  const u32 extents[3] = {batch, len, heads};
  for (int i = 0; i < 3; ++i) {
    if (extents[i] == 1) *strides[i] = 8;                       // never multiplied by more than 0
    if (*strides[i] % 8) return PS_E_ALIGN;
    if (*strides[i] == 0 || *strides[i] >= ((u64)1 << 38)) return PS_E_RANGE;
  }
  return PS_OK;
}

int ps_attention_forward(ps_ctx* ctx, const ps_attention_shape* shape, const ps_heads* q, const ps_heads* k,
                         const ps_heads* v, const ps_heads* out, float* d_lse, const int32_t* d_q_lens,
                         const int32_t* d_k_lens, void* d_work, uint64_t work_bytes) {
  if (!ctx || !shape) return PS_E_NULLPTR;
  AttentionArgs a;
  int rc = attention_args(*shape, a);
  if (rc != PS_OK) return rc;
  const ps_attention_shape& s = *shape;
  if ((rc = take_heads(q, s.batch, s.q_len, s.heads, a.q)) != PS_OK ||
      (rc = take_heads(k, s.batch, s.k_len, s.kv_heads, a.k)) != PS_OK ||
      (rc = take_heads(v, s.batch, s.k_len, s.kv_heads, a.v)) != PS_OK ||
      (rc = take_heads(out, s.batch, s.q_len, s.heads, a.out)) != PS_OK)
    return rc;
  if (s.batch == 0 || s.q_len == 0) return PS_OK;
  const u64 need = attention_forward_bytes(a);
  if (!d_lse || (need && !d_work)) return PS_E_NULLPTR;
  if (!aligned(d_lse, 4) || !aligned(d_q_lens, 4) || !aligned(d_k_lens, 4) || !aligned(d_work, 256)) return PS_E_ALIGN;
  if (work_bytes < need) return PS_E_RANGE;
  if ((rc = pending_device_error(ctx)) != PS_OK) return rc;
  DeviceGuard guard(ctx->device);
  if (!guard.ok) return PS_E_CUDA;
  a.lse = d_lse; a.q_lens = d_q_lens; a.k_lens = d_k_lens; a.status = ctx->h->status;
  a.work = d_work;
  CUDA_OK(launch_attention_forward(s.dtype, a, ctx->sm_count, ctx->stream));
  return PS_OK;
}

uint64_t ps_attention_forward_bytes(const ps_attention_shape* shape) {
  AttentionArgs a;
  return shape && attention_args(*shape, a) == PS_OK ? attention_forward_bytes(a) : 0;
}

uint64_t ps_attention_backward_bytes(const ps_attention_shape* shape) {
  AttentionArgs a;
  return shape && attention_args(*shape, a) == PS_OK ? attention_backward_bytes(a) : 0;
}

int ps_attention_backward(ps_ctx* ctx, const ps_attention_shape* shape, const ps_heads* q, const ps_heads* k,
                          const ps_heads* v, const ps_heads* out, const float* d_lse, const ps_heads* d_out,
                          const ps_heads* d_q, const ps_heads* d_k, const ps_heads* d_v, const int32_t* d_q_lens,
                          const int32_t* d_k_lens, void* d_work, uint64_t work_bytes) {
  if (!ctx || !shape) return PS_E_NULLPTR;
  AttentionArgs a;
  int rc = attention_args(*shape, a);
  if (rc != PS_OK) return rc;
  const ps_attention_shape& s = *shape;
  if ((rc = take_heads(q, s.batch, s.q_len, s.heads, a.q)) != PS_OK ||
      (rc = take_heads(k, s.batch, s.k_len, s.kv_heads, a.k)) != PS_OK ||
      (rc = take_heads(v, s.batch, s.k_len, s.kv_heads, a.v)) != PS_OK ||
      (rc = take_heads(out, s.batch, s.q_len, s.heads, a.out)) != PS_OK ||
      (rc = take_heads(d_out, s.batch, s.q_len, s.heads, a.d_out)) != PS_OK ||
      (rc = take_heads(d_q, s.batch, s.q_len, s.heads, a.d_q)) != PS_OK ||
      (rc = take_heads(d_k, s.batch, s.k_len, s.kv_heads, a.d_k)) != PS_OK ||
      (rc = take_heads(d_v, s.batch, s.k_len, s.kv_heads, a.d_v)) != PS_OK)
    return rc;
  if (s.batch == 0 || (s.q_len == 0 && s.k_len == 0)) return PS_OK;
  const u64 need = attention_backward_bytes(a);
  if ((s.q_len && !d_lse) || (need && !d_work)) return PS_E_NULLPTR;
  if (!aligned(d_lse, 4) || !aligned(d_q_lens, 4) || !aligned(d_k_lens, 4) || !aligned(d_work, 256)) return PS_E_ALIGN;
  if (work_bytes < need) return PS_E_RANGE;
  if ((rc = pending_device_error(ctx)) != PS_OK) return rc;
  DeviceGuard guard(ctx->device);
  if (!guard.ok) return PS_E_CUDA;
  a.lse = const_cast<float*>(d_lse); a.q_lens = d_q_lens; a.k_lens = d_k_lens; a.status = ctx->h->status;
  a.work = d_work;
  CUDA_OK(launch_attention_backward(s.dtype, a, ctx->sm_count, ctx->stream));
  return PS_OK;
}

// a matrix of the calls below: `step` is what its address and its rows' distance have to be multiples of, in elements
static int take_matrix(const ps_matrix* m, u64 rows, u64 cols, u64 width, u64 step, ps_matrix& into) {
  if (!m) return PS_E_NULLPTR;
  into = *m;
  if (rows == 0) return PS_OK;
  if (!m->data) return PS_E_NULLPTR;
  if (!aligned(m->data, step * width)) return PS_E_ALIGN;
  if (rows == 1) {
    into.stride = (cols + step - 1) / step * step;              // never multiplied by more than 0
    return PS_OK;
  }
  if (m->stride % step) return PS_E_ALIGN;
  if (m->stride < cols || m->stride > ((u64)1 << 40) / width / rows) return PS_E_RANGE;
  return PS_OK;
}
static int take_optional(const ps_matrix* m, u64 rows, u64 cols, u64 width, u64 step, ps_matrix& into) {
  into.data = nullptr, into.stride = 0;
  return m ? take_matrix(m, rows, cols, width, step, into) : PS_OK;
}
static int norm_args(const ps_layer_norm_desc& d, NormArgs& a) {
  if (d.rows > 0x7fffffffu || d.cols < 1 || d.cols > ((u64)1 << 20) || !(d.eps >= 0) || !std::isfinite((float)d.eps) || d.dtype > PS_F16 ||
      d.grad_dtype > PS_F16 || d.accumulate > 1)
    return PS_E_RANGE;
  memset(&a, 0, sizeof(a));
  a.rows = d.rows; a.cols = d.cols; a.eps = (float)d.eps;
  a.grad_dtype = d.grad_dtype; a.accumulate = d.accumulate;
  return PS_OK;
}

int ps_layer_norm_forward(ps_ctx* ctx, const ps_layer_norm_desc* desc, const ps_matrix* x, const void* d_weight, const void* d_bias,
                          const ps_matrix* y, float* d_mean, float* d_rstd) {
  if (!ctx || !desc) return PS_E_NULLPTR;
  NormArgs a;
  int rc = norm_args(*desc, a);
  if (rc != PS_OK) return rc;
  const u64 width = desc->dtype == PS_F32 ? 4 : 2;
  if ((rc = take_matrix(x, a.rows, a.cols, width, 1, a.x)) != PS_OK || (rc = take_matrix(y, a.rows, a.cols, width, 1, a.y)) != PS_OK) return rc;
  if (!aligned(d_weight, width) || !aligned(d_bias, width) || !aligned(d_mean, 4) || !aligned(d_rstd, 4)) return PS_E_ALIGN;
  if (a.rows == 0) return PS_OK;
  const Region x_at(a.x, a.rows, a.cols, width), y_at(a.y, a.rows, a.cols, width), w_at(d_weight, a.cols, width), b_at(d_bias, a.cols, width),
      mean_at(d_mean, a.rows, 4), rstd_at(d_rstd, a.rows, 4);
  if ((!same_rows(a.y, a.x, a.rows) && meet(y_at, x_at)) || meets(y_at, {w_at, b_at, mean_at, rstd_at}) || meets(mean_at, {x_at, w_at, b_at, rstd_at}) ||
      meets(rstd_at, {x_at, w_at, b_at}))
    return PS_E_RANGE;
  if ((rc = pending_device_error(ctx)) != PS_OK) return rc;
  DeviceGuard guard(ctx->device);
  if (!guard.ok) return PS_E_CUDA;
  a.weight = d_weight; a.bias = d_bias; a.mean = d_mean; a.rstd = d_rstd; a.status = ctx->h->status;
  CUDA_OK(launch_norm_forward(desc->dtype, a, ctx->sm_count, ctx->stream));
  return PS_OK;
}

uint64_t ps_layer_norm_backward_bytes(const ps_layer_norm_desc* desc) {
  NormArgs a;
  return desc && norm_args(*desc, a) == PS_OK ? norm_backward_bytes(desc->dtype, a) : 0;
}

int ps_layer_norm_backward(ps_ctx* ctx, const ps_layer_norm_desc* desc, const ps_matrix* y_grad, const ps_matrix* x, const float* d_mean,
                           const float* d_rstd, const void* d_weight, const ps_matrix* residual, const ps_matrix* x_grad, void* d_weight_grad,
                           void* d_bias_grad, void* d_work, uint64_t work_bytes) {
  if (!ctx || !desc) return PS_E_NULLPTR;
  NormArgs a;
  int rc = norm_args(*desc, a);
  if (rc != PS_OK) return rc;
  const u64 width = desc->dtype == PS_F32 ? 4 : 2, grad_width = desc->grad_dtype == PS_F32 ? 4 : 2;
  if ((rc = take_matrix(y_grad, a.rows, a.cols, width, 1, a.d_y)) != PS_OK || (rc = take_matrix(x, a.rows, a.cols, width, 1, a.x)) != PS_OK ||
      (rc = take_optional(residual, a.rows, a.cols, width, 1, a.residual)) != PS_OK ||
      (rc = take_matrix(x_grad, a.rows, a.cols, width, 1, a.d_x)) != PS_OK)
    return rc;
  const bool sums = d_weight_grad || d_bias_grad;
  const u64 need = sums ? norm_backward_bytes(desc->dtype, a) : 0;
  if ((a.rows && (!d_mean || !d_rstd)) || (need && !d_work)) return PS_E_NULLPTR;
  if (!aligned(d_weight, width) || !aligned(d_mean, 4) || !aligned(d_rstd, 4) || !aligned(d_weight_grad, grad_width) ||
      !aligned(d_bias_grad, grad_width) || !aligned(d_work, 256))
    return PS_E_ALIGN;
  if (work_bytes < need) return PS_E_RANGE;
  // (the gradients of weight and bias are written when everything else has been read)
  const auto rows_at = [&](const ps_matrix& m) { return Region(m, a.rows, a.cols, width); };
  const Region dx_at = rows_at(a.d_x), dw_at(d_weight_grad, a.cols, grad_width), db_at(d_bias_grad, a.cols, grad_width);
  for (const ps_matrix* m : {&a.d_y, &a.x, &a.residual})
    if (!same_rows(a.d_x, *m, a.rows) && meet(dx_at, rows_at(*m))) return PS_E_RANGE;
  if (meets(dx_at, {Region(d_weight, a.cols, width), Region(d_mean, a.rows, 4), Region(d_rstd, a.rows, 4), dw_at, db_at}) || meet(dw_at, db_at)) return PS_E_RANGE;
  if (a.rows == 0 && !sums) return PS_OK;
  if ((rc = pending_device_error(ctx)) != PS_OK) return rc;
  DeviceGuard guard(ctx->device);
  if (!guard.ok) return PS_E_CUDA;
  a.weight = d_weight; a.mean = const_cast<float*>(d_mean); a.rstd = const_cast<float*>(d_rstd);
  a.d_weight = d_weight_grad; a.d_bias = d_bias_grad;
  a.parts = sums ? (float*)d_work : nullptr;
  a.status = ctx->h->status;
  CUDA_OK(launch_norm_backward(desc->dtype, a, ctx->sm_count, ctx->stream));
  return PS_OK;
}

// heads of rotary positions: any alignment of the type, any strides; those that are written have none of 0
static int take_any_heads(const ps_heads* h, u32 batch, u32 len, u32 heads, u64 width, bool written, ps_heads& into) {
  if (!h || !h->data) return PS_E_NULLPTR;
  if (!aligned(h->data, width)) return PS_E_ALIGN;
  into = *h;
  u64* strides[3] = {&into.batch_stride, &into.token_stride, &into.head_stride};
  const u32 extents[3] = {batch, len, heads};
  for (int i = 0; i < 3; ++i) {
    if (extents[i] == 1) *strides[i] = 0;
    else if ((written && *strides[i] == 0) || *strides[i] >= ((u64)1 << 38)) return PS_E_RANGE;
  }
  return PS_OK;
}

int ps_rotary(ps_ctx* ctx, const ps_rotary_desc* desc, const ps_heads* q, const ps_heads* q_out, const ps_heads* k, const ps_heads* k_out,
              const void* d_positions) {
  if (!ctx || !desc) return PS_E_NULLPTR;
  const ps_rotary_desc& d = *desc;
  if (d.batch > 65535 || d.len > (1u << 24) || d.heads < 1 || d.heads > 32768 || d.kv_heads > 32768 || d.dim < 2 || d.dim > 256 ||
      d.rotary_dim < 2 || d.rotary_dim > d.dim || d.rotary_dim % 2 || d.dtype > PS_F16 || d.interleaved > 1 || d.inverse > 1 ||
      (d.position_bytes != 4 && d.position_bytes != 8) || d.position_stride > ((u64)1 << 38) ||
      (u64)d.batch * d.len * (d.heads + d.kv_heads) > ((u64)1 << 38))
    return PS_E_RANGE;
  if (!(d.base >= 1) || !std::isfinite(d.base) || !(d.factor >= 1) || !std::isfinite(d.factor) || !(d.original >= 0) || !std::isfinite(d.original) ||
      !std::isfinite(d.low) || !std::isfinite(d.high) || (d.original > 0 && d.factor != 1 && !(d.low < d.high)) || !std::isfinite((float)d.magnitude))
    return PS_E_RANGE;
  if (d.batch == 0 || d.len == 0) return PS_OK;
  RotaryArgs a;
  memset(&a, 0, sizeof(a));
  const u64 width = d.dtype == PS_F32 ? 4 : 2;
  int rc;
  if ((rc = take_any_heads(q, d.batch, d.len, d.heads, width, false, a.q)) != PS_OK ||
      (rc = take_any_heads(q_out, d.batch, d.len, d.heads, width, true, a.q_out)) != PS_OK)
    return rc;
  if (d.kv_heads && ((rc = take_any_heads(k, d.batch, d.len, d.kv_heads, width, false, a.k)) != PS_OK ||
                     (rc = take_any_heads(k_out, d.batch, d.len, d.kv_heads, width, true, a.k_out)) != PS_OK))
    return rc;
  if (!aligned(d_positions, d.position_bytes)) return PS_E_ALIGN;
  const auto same = [](const ps_heads& x, const ps_heads& y) {
    return x.data == y.data && x.batch_stride == y.batch_stride && x.token_stride == y.token_stride && x.head_stride == y.head_stride;
  };
  const auto heads_at = [&](const ps_heads& h, u32 heads) { return Region(h, d.batch, d.len, heads, d.dim, width); };
  const Region q_at = heads_at(a.q, d.heads), q_out_at = heads_at(a.q_out, d.heads), k_at = heads_at(a.k, d.kv_heads), k_out_at = heads_at(a.k_out, d.kv_heads);
  Region at_at(d_positions, d.len, d.position_bytes);
  at_at.along(0, d.position_stride * d.position_bytes, d.batch);
  if (meets(q_out_at, {k_at, k_out_at, at_at}) || meets(k_out_at, {q_at, at_at}) || (!same(a.q, a.q_out) && meet(q_out_at, q_at)) ||
      (!same(a.k, a.k_out) && meet(k_out_at, k_at)) || meets_itself(q_out_at) || meets_itself(k_out_at))
    return PS_E_RANGE;
  if ((rc = pending_device_error(ctx)) != PS_OK) return rc;
  DeviceGuard guard(ctx->device);
  if (!guard.ok) return PS_E_CUDA;
  a.positions = d_positions; a.position_stride = d.position_stride; a.position_bytes = d.position_bytes; a.first = d.first;
  a.batch = d.batch; a.len = d.len; a.heads = d.heads; a.kv_heads = d.kv_heads; a.dim = d.dim; a.pairs = d.rotary_dim / 2;
  a.interleaved = d.interleaved; a.inverse = d.inverse; a.magnitude = (float)d.magnitude;
  // The frequencies, one from the other: 128 products in 64 bits of mantissa are off by less than 2^-56.
  const long double turn = 6.283185307179586476925286766559L, step = powl((long double)d.base, -1.0L / a.pairs);
  long double f = 1.0L;
  for (u32 i = 0; i < a.pairs; ++i, f *= step) {
    long double g = f;
    if (d.factor != 1) {
      long double s = 0;
      if (d.original > 0) s = std::min(1.0L, std::max(0.0L, (d.original * f / turn - d.low) / ((long double)d.high - d.low)));
      g = f * (s + (1 - s) / d.factor);
    }
    a.turns[i] = (u64)(g / turn * 18446744073709551616.0L + 0.5L);
  }
  CUDA_OK(launch_rotary(d.dtype, a, ctx->sm_count, ctx->stream));
  return PS_OK;
}

static int linear_args(const ps_linear_desc& d, LinearArgs& a) {
  if (d.tokens > ((u64)1 << 30) || d.inputs < 1 || d.inputs > ((u64)1 << 24) || d.outputs < 1 || d.outputs > ((u64)1 << 24) ||
      (d.dtype != PS_BF16 && d.dtype != PS_F16) || (d.grad_dtype != d.dtype && d.grad_dtype != PS_F32) || d.activation > PS_ACT_SILU ||
      d.below_activation > PS_ACT_SILU || d.accumulate > 1)
    return PS_E_RANGE;
  if (d.tokens * std::max(d.inputs, d.outputs) > ((u64)1 << 39) || d.inputs * d.outputs > ((u64)1 << 38)) return PS_E_RANGE;
  memset(&a, 0, sizeof(a));
  a.tokens = d.tokens; a.inputs = d.inputs; a.outputs = d.outputs;
  a.dtype = d.dtype; a.grad_dtype = d.grad_dtype; a.activation = d.activation; a.below_activation = d.below_activation;
  a.accumulate = d.accumulate;
  return PS_OK;
}

int ps_linear_forward(ps_ctx* ctx, const ps_linear_desc* desc, const ps_matrix* x, const ps_matrix* weight, const void* d_bias,
                      const ps_matrix* residual, const ps_matrix* y, const ps_matrix* pre) {
  if (!ctx || !desc) return PS_E_NULLPTR;
  LinearArgs a;
  int rc = linear_args(*desc, a);
  if (rc != PS_OK) return rc;
  if ((rc = take_matrix(x, a.tokens, a.inputs, 2, 8, a.x)) != PS_OK || (rc = take_matrix(weight, a.outputs, a.inputs, 2, 8, a.weight)) != PS_OK ||
      (rc = take_optional(residual, a.tokens, a.outputs, 2, 8, a.residual)) != PS_OK ||
      (rc = take_matrix(y, a.tokens, a.outputs, 2, 8, a.y)) != PS_OK || (rc = take_optional(pre, a.tokens, a.outputs, 2, 8, a.pre)) != PS_OK)
    return rc;
  if (!aligned(d_bias, 2)) return PS_E_ALIGN;
  if (a.tokens == 0) return PS_OK;
  const Region x_at(a.x, a.tokens, a.inputs, 2), w_at(a.weight, a.outputs, a.inputs, 2), b_at(d_bias, a.outputs, 2),
      r_at(a.residual, a.tokens, a.outputs, 2), y_at(a.y, a.tokens, a.outputs, 2), pre_at(a.pre, a.tokens, a.outputs, 2);
  if (meets(y_at, {x_at, w_at, b_at, pre_at}) || meets(pre_at, {x_at, w_at, b_at, r_at}) ||
      (!same_rows(a.y, a.residual, a.tokens) && meet(y_at, r_at)))
    return PS_E_RANGE;
  if ((rc = pending_device_error(ctx)) != PS_OK) return rc;
  DeviceGuard guard(ctx->device);
  if (!guard.ok) return PS_E_CUDA;
  a.bias = d_bias; a.status = ctx->h->status;
  CUDA_OK(launch_linear_forward(a, ctx->sm_count, ctx->stream));
  return PS_OK;
}

uint64_t ps_linear_backward_bytes(const ps_linear_desc* desc) {
  LinearArgs a;
  return desc && linear_args(*desc, a) == PS_OK ? linear_backward_bytes(a) : 0;
}

int ps_linear_backward(ps_ctx* ctx, const ps_linear_desc* desc, const ps_matrix* y_grad, const ps_matrix* x, const ps_matrix* weight,
                       const ps_matrix* pre, const ps_matrix* below, const ps_matrix* residual, const ps_matrix* x_grad,
                       const ps_matrix* weight_grad, void* d_bias_grad, void* d_work, uint64_t work_bytes) {
  if (!ctx || !desc) return PS_E_NULLPTR;
  LinearArgs a;
  int rc = linear_args(*desc, a);
  if (rc != PS_OK) return rc;
  const u64 grad_width = desc->grad_dtype == PS_F32 ? 4 : 2;
  if ((rc = take_matrix(y_grad, a.tokens, a.outputs, 2, 8, a.d_y)) != PS_OK) return rc;
  // (what a result needs is looked at only where that result is wanted)
  if (a.activation && (rc = take_matrix(pre, a.tokens, a.outputs, 2, 8, a.pre)) != PS_OK) return rc;
  if (x_grad && ((rc = take_matrix(weight, a.outputs, a.inputs, 2, 8, a.weight)) != PS_OK ||
                 (a.below_activation && (rc = take_matrix(below, a.tokens, a.inputs, 2, 8, a.below)) != PS_OK) ||
                 (rc = take_optional(residual, a.tokens, a.inputs, 2, 8, a.residual)) != PS_OK ||
                 (rc = take_matrix(x_grad, a.tokens, a.inputs, 2, 8, a.d_x)) != PS_OK))
    return rc;
  if (weight_grad && ((rc = take_matrix(x, a.tokens, a.inputs, 2, 8, a.x)) != PS_OK ||
                      (rc = take_matrix(weight_grad, a.outputs, a.inputs, grad_width, 16 / grad_width, a.d_weight)) != PS_OK))
    return rc;
  const u64 need = linear_backward_bytes(a);
  if (need && !d_work) return PS_E_NULLPTR;
  if (!aligned(d_bias_grad, grad_width) || !aligned(d_work, 256)) return PS_E_ALIGN;
  if (work_bytes < need) return PS_E_RANGE;
  // (pre has been read before a product's result is written)
  const Region y_at(a.d_y, a.tokens, a.outputs, 2), x_at(a.x, a.tokens, a.inputs, 2), w_at(a.weight, a.outputs, a.inputs, 2),
      pre_at(a.pre, a.tokens, a.outputs, 2), below_at(a.below, a.tokens, a.inputs, 2), r_at(a.residual, a.tokens, a.inputs, 2),
      dx_at(a.d_x, a.tokens, a.inputs, 2), dw_at(a.d_weight, a.outputs, a.inputs, grad_width), db_at(d_bias_grad, a.outputs, grad_width);
  if (meets(dx_at, {y_at, x_at, w_at, dw_at, db_at}) || meets(dw_at, {y_at, x_at, w_at, below_at, r_at, db_at}) ||
      meets(db_at, {y_at, x_at, w_at, pre_at, below_at, r_at}) || (!same_rows(a.d_x, a.residual, a.tokens) && meet(dx_at, r_at)) ||
      (!same_rows(a.d_x, a.below, a.tokens) && meet(dx_at, below_at)))
    return PS_E_RANGE;
  if (!x_grad && !weight_grad && !d_bias_grad) return PS_OK;
  if ((rc = pending_device_error(ctx)) != PS_OK) return rc;
  DeviceGuard guard(ctx->device);
  if (!guard.ok) return PS_E_CUDA;
  if (!x_grad || a.tokens == 0) a.d_x.data = nullptr;
  a.d_bias = d_bias_grad; a.work = d_work; a.status = ctx->h->status;
  CUDA_OK(launch_linear_backward(a, ctx->sm_count, ctx->stream));
  return PS_OK;
}

// ------------------------------------------------------------------ measurement
int ps_int_peak(ps_ctx* ctx, uint32_t blocks, uint32_t iters, uint32_t* d_sink, uint64_t* thread_ops) {
  if (!ctx || !d_sink || !thread_ops) return PS_E_NULLPTR;
  if (blocks < 1 || blocks > (1u << 20) || iters < 1) return PS_E_RANGE;
  DeviceGuard guard(ctx->device);
  if (!guard.ok) return PS_E_CUDA;
  CUDA_OK(launch_int_peak(blocks, iters, d_sink, ctx->stream));
  *thread_ops = (u64)blocks * 256 * iters * 128;   // 8 rounds x 8 chains x 2 operations
  return PS_OK;
}

}  // extern "C"
