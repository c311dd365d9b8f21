// AdamW over many tensors at once (include/mtdao_ops.h).
//
// One launch takes every tensor: a workgroup owns a chunk of 4096 elements of
// one tensor, which a table of one word per chunk names.  A lane owns four (or,
// with bf16 parameters and 8-bit states, eight) consecutive elements of each slot,
// so that its accesses are 4 to 16 bytes and a wave's lie together; an 8-bit
// block of 128 lies in 32 (16) lanes, which form its new scale among themselves.
// All loads of a chunk are issued before the first is used.
//
// The pass is bound by HBM.  Bytes an element: fp32 states, parameters and
// gradients 28, 8-bit states 14 + 1/32 with fp32 parameters and bf16 gradients,
// 10 + 1/32 with bf16 parameters.  Nothing is read again soon, so loads and stores
// are non-temporal (354 M elements of 28 bytes 1821 -> 1700 us).  With 8-bit
// states the arithmetic is close behind: square root and quotient are the
// hardware's, an ulp each (IEEE sequences: 1311 M elements of 10 bytes 2750 us,
// 4.8 TB/s, against 2270 us), beta1 is folded into the blocks' scales (powers of
// two: no rounding more; a root of v has four significant bits, so its square
// rounds nothing either), and what only rare values need is behind branches
// (2180 us, 6.0 TB/s).

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstring>
#include <new>
#include <string>
#include <utility>
#include <vector>

#include "../../include/mtdao_ops.h"
#include "host.hpp"
#include "ops_device.hpp"

using namespace mtdao;
using namespace mtdao::ops;

namespace {

constexpr int kThreads = 256;
constexpr int kChunk = 4096;                 // elements of a workgroup
constexpr int kRowsAtOnce = 40;              // table rows that one launch's arguments carry

// A tensor's row of the device table.
struct Row {
  void* p;
  const void* g;
  void* m;
  void* v;
  uint8_t* ms;
  uint8_t* vs;
  int64_t numel;
  int64_t first;  // its first chunk
  float decay;    // weight decay
  float pad;
};

struct Rows {
  Row row[kRowsAtOnce];
};

struct Step {
  const Row* rows;
  const uint32_t* owner;   // tensor of every chunk
  const float* clip;       // the factor of the gradients (clipping)
  int64_t chunks;
  float beta1, rest1, beta2, rest2;  // rest = 1 - beta
  float lr, step;          // step = lr / (1 - beta1^t)
  float root2, eps;        // root2 = 1 / sqrt(1 - beta2^t)
  bool spread;             // Span
};

// The elements of a chunk.  Contiguous, or, in a spread pass, eight whole
// chunks share their span: each takes one piece of 64 lanes' elements in eight.
struct Span {
  int64_t base, left;
  bool spread;
};
template <int V>
__device__ __forceinline__ Span span_of(bool spread, int64_t c, int64_t numel) {
  const int64_t group = c & ~INT64_C(7);
  if (spread && (group + 8) * kChunk <= numel) return {group * kChunk + (c & 7) * (64 * V), INT64_MAX, true};
  return {c * kChunk, numel - c * kChunk, false};
}
// First element of a lane's slot from the span's base.
template <int V>
__device__ __forceinline__ int at_slot(int k, bool spread) {
  const int wave = (int)threadIdx.x >> 6, lane = (int)threadIdx.x & 63;
  const int piece = k * (kThreads / 64) + wave;
  return (spread ? 8 * piece : piece) * (64 * V) + lane * V;
}

__device__ __forceinline__ int64_t this_chunk() { return (int64_t)blockIdx.y * gridDim.x + blockIdx.x; }

// Writes rows `at`.. of the table and the owners of their chunks.
__global__ __launch_bounds__(kThreads) void k_adamw_table(Rows in, int at, Row* rows, uint32_t* owner) {
  const Row r = in.row[blockIdx.y];
  if (blockIdx.x == 0 && threadIdx.x == 0) rows[at + blockIdx.y] = r;
  const int64_t n = (r.numel + kChunk - 1) / kChunk;
  for (int64_t c = (int64_t)blockIdx.x * kThreads + threadIdx.x; c < n; c += (int64_t)gridDim.x * kThreads)
    owner[r.first + c] = (uint32_t)(at + blockIdx.y);
}

struct Grads {
  const void* g[4 * kRowsAtOnce];
};
__global__ __launch_bounds__(kThreads) void k_adamw_grads(Grads in, int at, int n, Row* rows) {
  if ((int)threadIdx.x < n) rows[at + threadIdx.x].g = in.g[threadIdx.x];
}

// ------------------------------------------------------------ gradient norm

template <typename GT>
__global__ __launch_bounds__(kThreads) void k_adamw_norm(const Row* rows, const uint32_t* owner, int64_t chunks,
                                                         double* partial) {
  __shared__ double part[kThreads / 64];
  const int64_t c = this_chunk();
  if (c >= chunks) return;
  const uint32_t t = uniform_load(owner + c);
  const GT* g = reinterpret_cast<const GT*>(uniform_load(&rows[t].g));
  constexpr int V = 4, kSlots = kChunk / (kThreads * V);
  const int64_t base = (c - uniform_load(&rows[t].first)) * kChunk, left = uniform_load(&rows[t].numel) - base;
  float a[kSlots][V];
#pragma unroll
  for (int s = 0; s < kSlots; ++s) {
    const int e = at_slot<V>(s, false);
    load_some<V>(g + base + e, left - e > V ? V : (int)(left - e), a[s]);
  }
  double sum = 0.0;
#pragma unroll
  for (int s = 0; s < kSlots; ++s)
#pragma unroll
    for (int k = 0; k < V; ++k) sum += (double)a[s][k] * (double)a[s][k];
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o);
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = sum;
  __syncthreads();
  if (threadIdx.x == 0) partial[c] = (part[0] + part[1]) + (part[2] + part[3]);
}

// The clip factor from the partial sums, each thread in steps of the block with
// several loads in flight (one by one: 36 us for 354 M elements, sixteen: 17 us).
constexpr int kFinish = 1024;
__global__ __launch_bounds__(kFinish) void k_adamw_clip(const double* partial, int64_t n, double max_norm, float* clip) {
  __shared__ double part[kFinish / 64];
  constexpr int kAtOnce = 16;
  double sum = 0.0;
  int64_t i = threadIdx.x;
  for (; i + (kAtOnce - 1) * kFinish < n; i += kAtOnce * kFinish) {
    double part_of[kAtOnce];
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k) part_of[k] = partial[i + k * kFinish];
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k) sum += part_of[k];
  }
  for (; i < n; i += kFinish) sum += partial[i];
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o);
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = sum;
  __syncthreads();
  if (threadIdx.x == 0) {
    sum = 0.0;
    for (int w = 0; w < kFinish / 64; ++w) sum += part[w];
    const double norm = sqrt(sum);
    *clip = norm > max_norm ? (float)(max_norm / norm) : norm == norm ? 1.0f : (float)norm;
  }
}

// --------------------------------------------------------------------- step

// V = 4 or 8 codes of a state.
template <int V>
struct Codes {
  typedef uint32_t Words __attribute__((ext_vector_type(V / 4)));
  uint32_t w[V / 4];
  __device__ __forceinline__ void load(const uint8_t* p, int n) {
    if (n >= V) {
      const Words a = vec_load<true, Words>(p);
#pragma unroll
      for (int i = 0; i < V / 4; ++i) w[i] = a[i];
    } else {
#pragma unroll
      for (int i = 0; i < V / 4; ++i) w[i] = 0;
#pragma unroll
      for (int t = 0; t < V; ++t)
        if (t < n) w[t / 4] |= (uint32_t)p[t] << (8 * (t % 4));
    }
  }
  __device__ __forceinline__ void store(uint8_t* p, int n) const {
    if (n >= V) {
      Words a;
#pragma unroll
      for (int i = 0; i < V / 4; ++i) a[i] = w[i];
      vec_store<true, Words>(p, a);
    } else {
#pragma unroll
      for (int t = 0; t < V; ++t)
        if (t < n) p[t] = (uint8_t)(w[t / 4] >> (8 * (t % 4)));
    }
  }
  __device__ __forceinline__ void values(float (&o)[V]) const {
#pragma unroll
    for (int i = 0; i < V / 4; ++i) {
      float a[4];
      values_of(w[i], a);
#pragma unroll
      for (int t = 0; t < 4; ++t) o[4 * i + t] = a[t];
    }
  }
  __device__ __forceinline__ void of(const float (&o)[V]) {
#pragma unroll
    for (int i = 0; i < V / 4; ++i) w[i] = codes_of(o[4 * i], o[4 * i + 1], o[4 * i + 2], o[4 * i + 3]);
  }
};

// Square roots by the hardware, off by an ulp; it takes numbers below 2^-126 for
// zero, so those (and zeros, hence the branch) are scaled first.
template <int V>
__device__ __forceinline__ void roots(const float (&from)[V], float (&r)[V]) {
  float v[V], least = 1.0f;
#pragma unroll
  for (int t = 0; t < V; ++t) {
    v[t] = from[t];
    r[t] = __builtin_amdgcn_sqrtf(v[t]);
    least = fminf(least, v[t]);
  }
  if (least < 0x1p-126f) {
#pragma unroll
    for (int t = 0; t < V; ++t)
      if (v[t] < 0x1p-126f) r[t] = __builtin_amdgcn_sqrtf(v[t] * 0x1p64f) * 0x1p-32f;
  }
}

template <typename PT, typename GT, bool EIGHT>
__global__ __launch_bounds__(kThreads) void k_adamw_step(Step s) {
  constexpr int V = EIGHT && sizeof(PT) == 2 ? 8 : 4, kSlots = kChunk / (kThreads * V);
  const int64_t c = this_chunk();
  if (c >= s.chunks) return;
  const Row* row = s.rows + uniform_load(s.owner + c);
  const Span span = span_of<V>(s.spread, c - uniform_load(&row->first), uniform_load(&row->numel));
  PT* p = reinterpret_cast<PT*>(uniform_load(&row->p)) + span.base;
  const GT* g = reinterpret_cast<const GT*>(uniform_load(&row->g)) + span.base;
  const float keep = 1.0f - s.lr * uniform_load(&row->decay);
  const float clip = s.clip ? uniform_load(s.clip) : 1.0f;
  // p from the new m and r = sqrt(v), each off by an ulp of v_sqrt and v_rcp
  auto moved = [&](float p, float m, float r) {
    return fmaf(-s.step * m, __builtin_amdgcn_rcpf(fmaf(r, s.root2, s.eps)), p * keep);
  };
  float pa[kSlots][V], ga[kSlots][V];
  int at[kSlots], n[kSlots];
#pragma unroll
  for (int k = 0; k < kSlots; ++k) {
    at[k] = at_slot<V>(k, span.spread);
    n[k] = span.left - at[k] > V ? V : (int)(span.left - at[k]);
    load_some<V, true>(p + at[k], n[k], pa[k]);
    load_some<V, true>(g + at[k], n[k], ga[k]);
  }
  if constexpr (!EIGHT) {
    float* m = reinterpret_cast<float*>(uniform_load(&row->m)) + span.base;
    float* v = reinterpret_cast<float*>(uniform_load(&row->v)) + span.base;
    float ma[kSlots][V], va[kSlots][V];
#pragma unroll
    for (int k = 0; k < kSlots; ++k) {
      load_some<V, true>(m + at[k], n[k], ma[k]);
      load_some<V, true>(v + at[k], n[k], va[k]);
    }
#pragma unroll
    for (int k = 0; k < kSlots; ++k) {
#pragma unroll
      for (int t = 0; t < V; ++t) {
        const float g = ga[k][t] * clip;
        ma[k][t] = fmaf(s.rest1, g, s.beta1 * ma[k][t]);
        va[k][t] = fmaf(s.rest2 * g, g, s.beta2 * va[k][t]);
      }
      float r[V];
      roots(va[k], r);
#pragma unroll
      for (int t = 0; t < V; ++t) pa[k][t] = moved(pa[k][t], ma[k][t], r[t]);
      store_some<V, true>(p + at[k], n[k], pa[k]);
      store_some<V, true>(m + at[k], n[k], ma[k]);
      store_some<V, true>(v + at[k], n[k], va[k]);
    }
  } else {
    uint8_t* m = reinterpret_cast<uint8_t*>(uniform_load(&row->m)) + span.base;
    uint8_t* v = reinterpret_cast<uint8_t*>(uniform_load(&row->v)) + span.base;
    uint8_t* ms = uniform_load(&row->ms) + span.base / kBlock8;
    uint8_t* vs = uniform_load(&row->vs) + span.base / kBlock8;
    constexpr int kLanes = kBlock8 / V;  // of a block
    Codes<V> mc[kSlots], vc[kSlots];
    uint32_t mb[kSlots], vb[kSlots];
#pragma unroll
    for (int k = 0; k < kSlots; ++k) {
      mc[k].load(m + at[k], n[k]);
      vc[k].load(v + at[k], n[k]);
      mb[k] = vb[k] = 0;
      if (n[k] > 0) {
        mb[k] = ms[at[k] / kBlock8];
        vb[k] = vs[at[k] / kBlock8];
      }
    }
#pragma unroll
    for (int k = 0; k < kSlots; ++k) {
      float ma[V], ra[V];
      mc[k].values(ma);
      vc[k].values(ra);
      const float mk = s.beta1 * scale_of(mb[k]), vk = scale_of(vb[k]);
      float mm = 0.0f, vm = 0.0f;
#pragma unroll
      for (int t = 0; t < V; ++t) {
        const float g = ga[k][t] * clip, r = vk * ra[t];
        ma[t] = fmaf(s.rest1, g, mk * ma[t]);
        ra[t] = fmaf(s.rest2 * g, g, s.beta2 * (r * r));
      }
      roots(ra, ra);
#pragma unroll
      for (int t = 0; t < V; ++t) {
        pa[k][t] = moved(pa[k][t], ma[t], ra[t]);
        mm = max_abs(mm, ma[t]);
        vm = fmaxf(vm, ra[t]);
      }
      store_some<V, true>(p + at[k], n[k], pa[k]);
      if (is_infinite(mm) || is_infinite(vm)) {
        mm = vm = 0.0f;
#pragma unroll
        for (int t = 0; t < V; ++t) {
          mm = fmaxf(mm, finite_abs(ma[t]));
          vm = fmaxf(vm, finite_abs(ra[t]));
        }
      }
      // (lanes past the tensor hold zeros)
      const uint32_t mbyte = scale_byte(kLanes == 16 ? max16(mm) : max32(mm));
      const uint32_t vbyte = scale_byte(kLanes == 16 ? max16(vm) : max32(vm));
      const float mi = inverse_scale_of(mbyte), vi = inverse_scale_of(vbyte);
      float least = 1.0f, scaled[V];
#pragma unroll
      for (int t = 0; t < V; ++t) {
        ma[t] *= mi;
        scaled[t] = ra[t] * vi;
        least = fminf(least, scaled[t]);
      }
      // what would round to zero and is none takes the smallest code
      if (least <= 0x1p-10f) {
#pragma unroll
        for (int t = 0; t < V; ++t)
          if (ra[t] > 0.0f) scaled[t] = fmaxf(scaled[t], 0x1p-9f);
      }
      mc[k].of(ma);
      vc[k].of(scaled);
      mc[k].store(m + at[k], n[k]);
      vc[k].store(v + at[k], n[k]);
      if ((threadIdx.x & (kLanes - 1)) == 0 && n[k] > 0) {
        ms[at[k] / kBlock8] = (uint8_t)mbyte;
        vs[at[k] / kBlock8] = (uint8_t)vbyte;
      }
    }
  }
}

// --------------------------------------------------------------------- host

// Grids of one workgroup per chunk: x below 2^22 (2^30 threads).
dim3 chunk_grid(int64_t chunks) {
  const int64_t most = INT64_C(1) << 22, y = (chunks + most - 1) / most;
  return dim3((unsigned)((chunks + y - 1) / y), (unsigned)y);
}

int64_t chunks_of(int64_t numel) { return (numel + kChunk - 1) / kChunk; }
int64_t esize(int32_t dt) { return dt == MTDAO_BF16 ? 2 : 4; }
size_t up256(size_t n) { return (n + 255) / 256 * 256; }

// How a pass goes over its elements.  Workgroups of one CU and, for states of
// 32 bits, spread pieces set how many DRAM pages are open at once.  Measured for
// 354 M elements, all the registers allow and contiguous against the choice here:
// 32 bits, fp32 1688 -> 1643 us (6.0 TB/s; the rest of a chunk's 64 KiB of loads
// in two workgroups covers the latency), 32 bits with bf16 parameters and
// gradients 1283 -> 1226 us, four workgroups (two 1505 us); 8 bits with fp32
// parameters 839 -> 803 us, four workgroups, contiguous (spread 827 us).  In
// between, 32 bits: 256 M 1216 -> 1145 us (bf16 915 -> 880), 128 M 597 -> 577 (456
// -> 445), 64 M 294 -> 286 (232 -> 226).  Below 64 M they gain less than their noise
// or lose (48 M 223.5 and 223.4 us, 32 M 145.9 and 146.9, 8 M 36.3 and 40.0); with
// bf16 parameters 8-bit passes lose at any limit (1311 M: 2081 and 2202 us).  The
// limit is an amount of unused LDS, of 160 KiB.
struct Pass {
  bool spread;
  size_t lds;
};
Pass pass_of(const mtdao_adamw_config& c, int64_t elements) {
  constexpr size_t kTwo = 64 * 1024, kFour = 40 * 1024;
  if (c.state_bits == 8) return {false, c.param_dtype == MTDAO_F32 ? kFour : 0};
  if (elements < INT64_C(64) << 20) return {false, 0};
  return {true, c.param_dtype == MTDAO_F32 && c.grad_dtype == MTDAO_F32 ? kTwo : kFour};
}

struct Layout {
  size_t owner, partial, clip, bytes;
  int64_t chunks;
};

Layout layout_of(const mtdao_adamw_config& c, const mtdao_adamw_tensor* t) {
  Layout l;
  l.chunks = 0;
  for (int i = 0; i < c.n_tensors; ++i) l.chunks += chunks_of(t[i].numel);
  l.owner = up256((size_t)c.n_tensors * sizeof(Row));
  l.clip = l.owner + up256((size_t)l.chunks * sizeof(uint32_t));
  l.partial = l.clip + 256;
  l.bytes = c.max_norm > 0.0 ? l.partial + (size_t)l.chunks * sizeof(double) : l.clip;
  return l;
}

int32_t validate(const mtdao_adamw_config* c, const mtdao_adamw_tensor* t, std::string* e) {
  if (!c || !t) return fail(e, MTDAO_ERR_INVALID_ARG, "config or tensors is NULL");
  if ((c->param_dtype != MTDAO_F32 && c->param_dtype != MTDAO_BF16) ||
      (c->grad_dtype != MTDAO_F32 && c->grad_dtype != MTDAO_BF16))
    return fail(e, MTDAO_ERR_INVALID_ARG, "param_dtype/grad_dtype must be F32(0) or BF16(1)");
  if (c->state_bits != 32 && c->state_bits != 8)
    return fail(e, MTDAO_ERR_INVALID_ARG, "state_bits %d is not 32 or 8", c->state_bits);
  if (c->n_tensors < 1) return fail(e, MTDAO_ERR_INVALID_ARG, "n_tensors %d < 1", c->n_tensors);
  if (!(c->beta1 >= 0.0 && c->beta1 < 1.0) || !(c->beta2 >= 0.0 && c->beta2 < 1.0))
    return fail(e, MTDAO_ERR_INVALID_ARG, "beta1=%g, beta2=%g: both in [0,1)", c->beta1, c->beta2);
  if (!(c->eps >= 0.0) || !std::isfinite((float)c->eps))
    return fail(e, MTDAO_ERR_INVALID_ARG, "eps=%g must be finite and >= 0", c->eps);
  if (!std::isfinite(c->max_norm)) return fail(e, MTDAO_ERR_INVALID_ARG, "max_norm is not finite");
  if (c->start_step < 0) return fail(e, MTDAO_ERR_INVALID_ARG, "start_step < 0");
  int64_t sum = 0;
  for (int i = 0; i < c->n_tensors; ++i) {
    if (t[i].numel < 0) return fail(e, MTDAO_ERR_INVALID_ARG, "numel of tensor %d < 0", i);
    if (t[i].numel > (INT64_C(1) << 40) - sum)
      return fail(e, MTDAO_ERR_INVALID_ARG, "the tensors exceed 2^40 elements");
    sum += t[i].numel;
    if (!(t[i].weight_decay >= 0.0) || !std::isfinite((float)t[i].weight_decay))
      return fail(e, MTDAO_ERR_INVALID_ARG, "weight_decay of tensor %d must be finite and >= 0", i);
  }
  return MTDAO_OK;
}

// Memory that steps write: [lo, hi) of a tensor.
struct Written {
  uintptr_t lo, hi;
  int tensor;
};

// written: in order, none over another.  A gradient may lie on its own tensor's
// parameters or states, element on element: a lane reads all of its elements
// before it writes them.  Elsewhere it would be read while it changes.
int32_t check_grad(const mtdao_adamw_config& c, int i, int64_t numel, const void* g, const std::vector<Written>& written, std::string* e) {
  if (numel == 0) return MTDAO_OK;
  if (!g) return fail(e, MTDAO_ERR_INVALID_ARG, "g of tensor %d is NULL", i);
  if (!aligned_to(g, (uintptr_t)esize(c.grad_dtype)))
    return fail(e, MTDAO_ERR_ALIGN, "g of tensor %d is not aligned to its element", i);
  const uintptr_t lo = (uintptr_t)g, hi = lo + (uintptr_t)(numel * esize(c.grad_dtype));
  auto w = std::upper_bound(written.begin(), written.end(), lo, [](uintptr_t at, const Written& r) { return at < r.hi; });
  for (; w != written.end() && w->lo < hi; ++w)
    if (w->tensor != i || w->lo != lo || w->hi != hi)
      return fail(e, MTDAO_ERR_INVALID_ARG, "g of tensor %d overlaps parameters or states of tensor %d", i, w->tensor);
  return MTDAO_OK;
}

int32_t check_pointers(const mtdao_adamw_config& c, const mtdao_adamw_tensor* t, std::vector<Written>& written, std::string* e) {
  const bool eight = c.state_bits == 8;
  for (int i = 0; i < c.n_tensors; ++i) {
    const mtdao_adamw_tensor& a = t[i];
    if (a.numel == 0) continue;
    if (!a.p || !a.m || !a.v) return fail(e, MTDAO_ERR_INVALID_ARG, "p, m or v of tensor %d is NULL", i);
    if (eight && (!a.m_scale || !a.v_scale))
      return fail(e, MTDAO_ERR_INVALID_ARG, "m_scale or v_scale of tensor %d is NULL", i);
    if (!aligned_to(a.p, (uintptr_t)esize(c.param_dtype)))
      return fail(e, MTDAO_ERR_ALIGN, "p of tensor %d is not aligned to its element", i);
    if (!aligned16(a.m) || !aligned16(a.v)) return fail(e, MTDAO_ERR_ALIGN, "m or v of tensor %d is not 16-byte aligned", i);
    auto add = [&](const void* p, int64_t bytes) { written.push_back({(uintptr_t)p, (uintptr_t)p + (uintptr_t)bytes, i}); };
    const int64_t blocks = (a.numel + kBlock8 - 1) / kBlock8;
    add(a.p, a.numel * esize(c.param_dtype));
    add(a.m, a.numel * (eight ? 1 : 4));
    add(a.v, a.numel * (eight ? 1 : 4));
    if (eight) {
      add(a.m_scale, blocks);
      add(a.v_scale, blocks);
    }
  }
  std::sort(written.begin(), written.end(), [](const Written& x, const Written& y) { return x.lo < y.lo; });
  for (size_t k = 1; k < written.size(); ++k)
    if (written[k].lo < written[k - 1].hi)
      return fail(e, MTDAO_ERR_INVALID_ARG, "parameters or states of the tensors overlap");
  for (int i = 0; i < c.n_tensors; ++i) {
    const int32_t r = check_grad(c, i, t[i].numel, t[i].g, written, e);
    if (r != MTDAO_OK) return r;
  }
  return MTDAO_OK;
}

}  // namespace

struct mtdao_adamw {
  mtdao_adamw_config cfg;
  std::vector<int64_t> numel;
  std::vector<Written> written;
  Row* rows = nullptr;
  uint32_t* owner = nullptr;
  float* clip = nullptr;
  double* partial = nullptr;
  int64_t chunks = 0;
  int64_t elements = 0;
  int64_t t = 0;
  std::string err;
};

extern "C" {

int32_t mtdao_adamw_workspace_bytes(const mtdao_adamw_config* cfg, const mtdao_adamw_tensor* tensors, size_t* bytes) {
  const int32_t r = validate(cfg, tensors, &g_err);
  if (r != MTDAO_OK) return r;
  if (!bytes) return fail(&g_err, MTDAO_ERR_INVALID_ARG, "bytes is NULL");
  *bytes = layout_of(*cfg, tensors).bytes;
  return MTDAO_OK;
}

int32_t mtdao_adamw_init(const mtdao_adamw_config* cfg, const mtdao_adamw_tensor* tensors, void* workspace,
                         size_t workspace_bytes, void* hip_stream, mtdao_adamw** out) try {
  int32_t r = validate(cfg, tensors, &g_err);
  if (r != MTDAO_OK) return r;
  if (!out) return fail(&g_err, MTDAO_ERR_INVALID_ARG, "out is NULL");
  const mtdao_adamw_config& c = *cfg;
  std::vector<Written> written;
  r = check_pointers(c, tensors, written, &g_err);
  if (r != MTDAO_OK) return r;
  const Layout l = layout_of(c, tensors);
  if (!workspace || workspace_bytes < l.bytes)
    return fail(&g_err, MTDAO_ERR_WORKSPACE, "workspace of %zu bytes required, %zu given", l.bytes,
                workspace ? workspace_bytes : (size_t)0);
  if (!aligned_to(workspace, 256)) return fail(&g_err, MTDAO_ERR_ALIGN, "workspace is not 256-byte aligned");

  struct Owned {
    mtdao_adamw* h = new mtdao_adamw();
    ~Owned() { delete h; }
  } own;
  mtdao_adamw* h = own.h;
  char* w = static_cast<char*>(workspace);
  h->cfg = c;
  h->written = std::move(written);
  h->rows = reinterpret_cast<Row*>(w);
  h->owner = reinterpret_cast<uint32_t*>(w + l.owner);
  if (c.max_norm > 0.0) {
    h->clip = reinterpret_cast<float*>(w + l.clip);
    h->partial = reinterpret_cast<double*>(w + l.partial);
  }
  h->chunks = l.chunks;
  h->t = c.start_step;
  for (int i = 0; i < c.n_tensors; ++i) {
    h->numel.push_back(tensors[i].numel);
    h->elements += tensors[i].numel;
  }

  hipStream_t st = reinterpret_cast<hipStream_t>(hip_stream);
  RoctxRange range("mtdao_adamw_init tensors=%d", c.n_tensors);
  int64_t first = 0;
  for (int at = 0; at < c.n_tensors; at += kRowsAtOnce) {
    Rows in;
    std::memset(&in, 0, sizeof in);
    const int n = std::min(kRowsAtOnce, c.n_tensors - at);
    int64_t most = 0;
    for (int k = 0; k < n; ++k) {
      const mtdao_adamw_tensor& a = tensors[at + k];
      in.row[k] = {a.p, a.g, a.m, a.v, a.m_scale, a.v_scale, a.numel, first, (float)a.weight_decay, 0.0f};
      first += chunks_of(a.numel);
      most = std::max(most, chunks_of(a.numel));
    }
    const unsigned x = (unsigned)std::min<int64_t>(64, std::max<int64_t>(1, (most + kThreads - 1) / kThreads));
    hipLaunchKernelGGL(k_adamw_table, dim3(x, (unsigned)n), dim3(kThreads), 0, st, in, at, h->rows, h->owner);
  }
  r = hip_check(&g_err, hipGetLastError(), "mtdao_adamw_init launch");
  if (r != MTDAO_OK) return r;
  g_err.clear();
  *out = h;
  own.h = nullptr;
  return MTDAO_OK;
} catch (const std::bad_alloc&) {
  return fail(&g_err, MTDAO_ERR_WORKSPACE, "out of host memory");
}

int32_t mtdao_adamw_set_grads(mtdao_adamw* h, const void* const* grads, void* hip_stream) {
  if (!h) return fail(&g_err, MTDAO_ERR_INVALID_ARG, "handle is NULL");
  if (!grads) return fail(&h->err, MTDAO_ERR_INVALID_ARG, "grads is NULL");
  const int n = h->cfg.n_tensors;
  for (int i = 0; i < n; ++i) {
    const int32_t r = check_grad(h->cfg, i, h->numel[i], grads[i], h->written, &h->err);
    if (r != MTDAO_OK) return r;
  }
  hipStream_t st = reinterpret_cast<hipStream_t>(hip_stream);
  RoctxRange range("mtdao_adamw_set_grads tensors=%d", n);
  constexpr int most = 4 * kRowsAtOnce;
  for (int at = 0; at < n; at += most) {
    Grads in;
    std::memset(&in, 0, sizeof in);
    const int some = std::min(most, n - at);
    std::copy(grads + at, grads + at + some, in.g);
    hipLaunchKernelGGL(k_adamw_grads, dim3(1), dim3(kThreads), 0, st, in, at, some, h->rows);
  }
  return hip_check(&h->err, hipGetLastError(), "mtdao_adamw_set_grads launch");
}

int32_t mtdao_adamw_step(mtdao_adamw* h, double lr, void* hip_stream) {
  if (!h) return fail(&g_err, MTDAO_ERR_INVALID_ARG, "handle is NULL");
  if (!std::isfinite((float)lr)) return fail(&h->err, MTDAO_ERR_INVALID_ARG, "lr is not finite");
  const mtdao_adamw_config& c = h->cfg;
  const int64_t t = h->t + 1;
  hipStream_t st = reinterpret_cast<hipStream_t>(hip_stream);
  RoctxRange range("mtdao_adamw_step t=%lld", (long long)t);
  if (h->chunks > 0) {
    const dim3 grid = chunk_grid(h->chunks), block(kThreads);
    if (h->clip) {
      if (c.grad_dtype == MTDAO_F32)
        hipLaunchKernelGGL(k_adamw_norm<float>, grid, block, 0, st, h->rows, h->owner, h->chunks, h->partial);
      else
        hipLaunchKernelGGL(k_adamw_norm<bf16_t>, grid, block, 0, st, h->rows, h->owner, h->chunks, h->partial);
      hipLaunchKernelGGL(k_adamw_clip, dim3(1), dim3(kFinish), 0, st, h->partial, h->chunks, c.max_norm, h->clip);
    }
    Step s;
    s.rows = h->rows;
    s.owner = h->owner;
    s.clip = h->clip;
    s.chunks = h->chunks;
    s.beta1 = (float)c.beta1;
    s.rest1 = (float)(1.0 - c.beta1);
    s.beta2 = (float)c.beta2;
    s.rest2 = (float)(1.0 - c.beta2);
    const Pass pass = pass_of(c, h->elements);
    s.spread = pass.spread;
    s.lr = (float)lr;
    // m / (sqrt(v) + eps): both sides times a power of two where eps is close to the
    // numbers that the hardware's reciprocal takes for zero, which made NaN of m = v = 0
    const bool tiny = c.eps > 0.0 && c.eps < 0x1p-100;
    const double both = tiny ? 0x1p40 : 1.0;
    s.step = (float)(both * lr / (1.0 - std::pow(c.beta1, (double)t)));
    s.root2 = (float)(both / std::sqrt(1.0 - std::pow(c.beta2, (double)t)));
    s.eps = (float)(tiny ? std::max(both * c.eps, 0x1p-126) : c.eps);
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, block, pass.lds, st, s); };
    auto with = [&](auto p, auto g) {
      using PT = decltype(p);
      using GT = decltype(g);
      if (c.state_bits == 8) go(k_adamw_step<PT, GT, true>);
      else go(k_adamw_step<PT, GT, false>);
    };
    if (c.param_dtype == MTDAO_F32 && c.grad_dtype == MTDAO_F32) with(float{}, float{});
    else if (c.param_dtype == MTDAO_F32) with(float{}, bf16_t{});
    else if (c.grad_dtype == MTDAO_F32) with(bf16_t{}, float{});
    else with(bf16_t{}, bf16_t{});
    const int32_t r = hip_check(&h->err, hipGetLastError(), "mtdao_adamw_step launch");
    if (r != MTDAO_OK) return r;
  }
  h->t = t;
  return MTDAO_OK;
}

int64_t mtdao_adamw_step_count(const mtdao_adamw* h) { return h ? h->t : -1; }

const char* mtdao_adamw_last_error(const mtdao_adamw* h) { return h ? h->err.c_str() : g_err.c_str(); }

void mtdao_adamw_destroy(mtdao_adamw* h) { delete h; }

}  // extern "C"
