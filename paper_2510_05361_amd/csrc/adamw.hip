// AdamW over many tensors at once (include/mtdao_ops.h).
//
// One launch takes every tensor: a workgroup owns a chunk of kChunk
// consecutive elements of one tensor, which a table of one word per chunk
// names.  A lane owns four consecutive elements of each slot of 1024, so fp32
// accesses are 16 bytes a lane and 1 KiB a wave; an 8-bit block of 128 lies in
// 32 lanes, which form its new scale among themselves.  All loads of a chunk
// are issued before the first is used.  The pass is bound by HBM: fp32 states
// 28 bytes an element with fp32 parameters and gradients, 8-bit states
// 14 + 1/32 with fp32 parameters and bf16 gradients.

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
constexpr int kV = 4;                        // elements of a lane's slot
constexpr int kSlots = 4;                    // slots of a chunk
constexpr int kSlot = kThreads * kV;         // elements of a slot
constexpr int kChunk = kSlots * kSlot;       // 4096
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
};

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
  const int64_t base = (c - uniform_load(&rows[t].first)) * kChunk, left = uniform_load(&rows[t].numel) - base;
  float a[kSlots][kV];
#pragma unroll
  for (int s = 0; s < kSlots; ++s) {
    const int e = s * kSlot + (int)threadIdx.x * kV;
    load_some<kV>(g + base + e, left - e > kV ? kV : (int)(left - e), a[s]);
  }
  double sum = 0.0;
#pragma unroll
  for (int s = 0; s < kSlots; ++s)
#pragma unroll
    for (int k = 0; k < kV; ++k) sum += (double)a[s][k] * (double)a[s][k];
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o);
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = sum;
  __syncthreads();
  if (threadIdx.x == 0) partial[c] = (part[0] + part[1]) + (part[2] + part[3]);
}

// The clip factor from the partial sums, each thread in steps of the block.
constexpr int kFinish = 1024;
__global__ __launch_bounds__(kFinish) void k_adamw_clip(const double* partial, int64_t n, double max_norm, float* clip) {
  __shared__ double part[kFinish / 64];
  double sum = 0.0;
  for (int64_t i = threadIdx.x; i < n; i += kFinish) sum += partial[i];
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

// One slot: m, v from their stored values, p from the new ones.
__device__ __forceinline__ void update(const Step& s, float keep, const float (&g)[kV], float (&p)[kV], float (&m)[kV],
                                       float (&v)[kV]) {
#pragma unroll
  for (int k = 0; k < kV; ++k) {
    m[k] = fmaf(s.rest1, g[k], s.beta1 * m[k]);
    v[k] = fmaf(s.rest2 * g[k], g[k], s.beta2 * v[k]);
    const float r = sqrtf(v[k]);
    p[k] = fmaf(-s.step, m[k] / fmaf(r, s.root2, s.eps), p[k] * keep);
  }
}

template <typename PT, typename GT, bool EIGHT>
__global__ __launch_bounds__(kThreads) void k_adamw_step(Step s) {
  const int64_t c = this_chunk();
  if (c >= s.chunks) return;
  const Row* row = s.rows + uniform_load(s.owner + c);
  const int64_t base = (c - uniform_load(&row->first)) * kChunk, left = uniform_load(&row->numel) - base;
  PT* p = reinterpret_cast<PT*>(uniform_load(&row->p)) + base;
  const GT* g = reinterpret_cast<const GT*>(uniform_load(&row->g)) + base;
  const float keep = 1.0f - s.lr * uniform_load(&row->decay);
  const float clip = s.clip ? uniform_load(s.clip) : 1.0f;
  float pa[kSlots][kV], ga[kSlots][kV];
  int n[kSlots];
#pragma unroll
  for (int k = 0; k < kSlots; ++k) {
    const int e = k * kSlot + (int)threadIdx.x * kV;
    n[k] = left - e > kV ? kV : (int)(left - e);
    load_some<kV>(p + e, n[k], pa[k]);
    load_some<kV>(g + e, n[k], ga[k]);
  }
  if constexpr (!EIGHT) {
    float* m = reinterpret_cast<float*>(uniform_load(&row->m)) + base;
    float* v = reinterpret_cast<float*>(uniform_load(&row->v)) + base;
    float ma[kSlots][kV], va[kSlots][kV];
#pragma unroll
    for (int k = 0; k < kSlots; ++k) {
      const int e = k * kSlot + (int)threadIdx.x * kV;
      load_some<kV>(m + e, n[k], ma[k]);
      load_some<kV>(v + e, n[k], va[k]);
    }
#pragma unroll
    for (int k = 0; k < kSlots; ++k) {
      const int e = k * kSlot + (int)threadIdx.x * kV;
#pragma unroll
      for (int t = 0; t < kV; ++t) ga[k][t] *= clip;
      update(s, keep, ga[k], pa[k], ma[k], va[k]);
      store_some<kV>(p + e, n[k], pa[k]);
      store_some<kV>(m + e, n[k], ma[k]);
      store_some<kV>(v + e, n[k], va[k]);
    }
  } else {
    uint8_t* m = reinterpret_cast<uint8_t*>(uniform_load(&row->m)) + base;
    uint8_t* v = reinterpret_cast<uint8_t*>(uniform_load(&row->v)) + base;
    uint8_t* ms = uniform_load(&row->ms) + base / kBlock8;
    uint8_t* vs = uniform_load(&row->vs) + base / kBlock8;
    uint32_t mc[kSlots], vc[kSlots], mb[kSlots], vb[kSlots];
#pragma unroll
    for (int k = 0; k < kSlots; ++k) {
      const int e = k * kSlot + (int)threadIdx.x * kV;
      mc[k] = vc[k] = mb[k] = vb[k] = 0;
      if (n[k] >= kV) {
        mc[k] = *reinterpret_cast<const uint32_t*>(m + e);
        vc[k] = *reinterpret_cast<const uint32_t*>(v + e);
      } else {
#pragma unroll
        for (int t = 0; t < kV; ++t)
          if (t < n[k]) {
            mc[k] |= (uint32_t)m[e + t] << (8 * t);
            vc[k] |= (uint32_t)v[e + t] << (8 * t);
          }
      }
      if (n[k] > 0) {
        mb[k] = ms[e / kBlock8];
        vb[k] = vs[e / kBlock8];
      }
    }
#pragma unroll
    for (int k = 0; k < kSlots; ++k) {
      const int e = k * kSlot + (int)threadIdx.x * kV;
      float ma[kV], va[kV];
      values_of(mc[k], ma);
      values_of(vc[k], va);
      const float msc = scale_of(mb[k]), vsc = scale_of(vb[k]);
#pragma unroll
      for (int t = 0; t < kV; ++t) {
        ga[k][t] *= clip;
        ma[t] *= msc;
        va[t] *= vsc;
        va[t] *= va[t];
      }
      update(s, keep, ga[k], pa[k], ma, va);
      store_some<kV>(p + e, n[k], pa[k]);
      float mm = 0.0f, vm = 0.0f;
#pragma unroll
      for (int t = 0; t < kV; ++t) {
        va[t] = sqrtf(va[t]);
        mm = max_abs(mm, ma[t]);
        vm = max_abs(vm, va[t]);
      }
      if (is_infinite(mm) || is_infinite(vm)) {
        mm = vm = 0.0f;
#pragma unroll
        for (int t = 0; t < kV; ++t) {
          mm = fmaxf(mm, finite_abs(ma[t]));
          vm = fmaxf(vm, finite_abs(va[t]));
        }
      }
      // (lanes past the tensor hold zeros)
      const uint32_t mbyte = scale_byte(max32(mm)), vbyte = scale_byte(max32(vm));
      const float mi = inverse_scale_of(mbyte), vi = inverse_scale_of(vbyte);
#pragma unroll
      for (int t = 0; t < kV; ++t) {
        ma[t] *= mi;
        va[t] = va[t] > 0.0f ? fmaxf(va[t] * vi, 0x1p-9f) : va[t] * vi;
      }
      const uint32_t mq = codes_of(ma[0], ma[1], ma[2], ma[3]), vq = codes_of(va[0], va[1], va[2], va[3]);
      if (n[k] >= kV) {
        *reinterpret_cast<uint32_t*>(m + e) = mq;
        *reinterpret_cast<uint32_t*>(v + e) = vq;
      } else {
#pragma unroll
        for (int t = 0; t < kV; ++t)
          if (t < n[k]) {
            m[e + t] = (uint8_t)(mq >> (8 * t));
            v[e + t] = (uint8_t)(vq >> (8 * t));
          }
      }
      if ((threadIdx.x & 31) == 0 && n[k] > 0) {
        ms[e / kBlock8] = (uint8_t)mbyte;
        vs[e / kBlock8] = (uint8_t)vbyte;
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

int32_t check_grad(const mtdao_adamw_config& c, int i, int64_t numel, const void* g, std::string* e) {
  if (numel == 0) return MTDAO_OK;
  if (!g) return fail(e, MTDAO_ERR_INVALID_ARG, "g of tensor %d is NULL", i);
  if (!aligned_to(g, (uintptr_t)esize(c.grad_dtype)))
    return fail(e, MTDAO_ERR_ALIGN, "g of tensor %d is not aligned to its element", i);
  return MTDAO_OK;
}

int32_t check_pointers(const mtdao_adamw_config& c, const mtdao_adamw_tensor* t, std::string* e) {
  const bool eight = c.state_bits == 8;
  std::vector<std::pair<uintptr_t, uintptr_t>> written;
  for (int i = 0; i < c.n_tensors; ++i) {
    const mtdao_adamw_tensor& a = t[i];
    if (a.numel == 0) continue;
    if (!a.p || !a.m || !a.v) return fail(e, MTDAO_ERR_INVALID_ARG, "p, m or v of tensor %d is NULL", i);
    if (eight && (!a.m_scale || !a.v_scale))
      return fail(e, MTDAO_ERR_INVALID_ARG, "m_scale or v_scale of tensor %d is NULL", i);
    if (!aligned_to(a.p, (uintptr_t)esize(c.param_dtype)))
      return fail(e, MTDAO_ERR_ALIGN, "p of tensor %d is not aligned to its element", i);
    if (!aligned16(a.m) || !aligned16(a.v)) return fail(e, MTDAO_ERR_ALIGN, "m or v of tensor %d is not 16-byte aligned", i);
    const int32_t r = check_grad(c, i, a.numel, a.g, e);
    if (r != MTDAO_OK) return r;
    auto add = [&](const void* p, int64_t bytes) { written.push_back({(uintptr_t)p, (uintptr_t)p + (uintptr_t)bytes}); };
    const int64_t blocks = (a.numel + kBlock8 - 1) / kBlock8;
    add(a.p, a.numel * esize(c.param_dtype));
    add(a.m, a.numel * (eight ? 1 : 4));
    add(a.v, a.numel * (eight ? 1 : 4));
    if (eight) {
      add(a.m_scale, blocks);
      add(a.v_scale, blocks);
    }
  }
  std::sort(written.begin(), written.end());
  for (size_t k = 1; k < written.size(); ++k)
    if (written[k].first < written[k - 1].second)
      return fail(e, MTDAO_ERR_INVALID_ARG, "parameters or states of the tensors overlap");
  return MTDAO_OK;
}

}  // namespace

struct mtdao_adamw {
  mtdao_adamw_config cfg;
  std::vector<int64_t> numel;
  Row* rows = nullptr;
  uint32_t* owner = nullptr;
  float* clip = nullptr;
  double* partial = nullptr;
  int64_t chunks = 0;
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
  r = check_pointers(c, tensors, &g_err);
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
  h->rows = reinterpret_cast<Row*>(w);
  h->owner = reinterpret_cast<uint32_t*>(w + l.owner);
  if (c.max_norm > 0.0) {
    h->clip = reinterpret_cast<float*>(w + l.clip);
    h->partial = reinterpret_cast<double*>(w + l.partial);
  }
  h->chunks = l.chunks;
  h->t = c.start_step;
  for (int i = 0; i < c.n_tensors; ++i) h->numel.push_back(tensors[i].numel);

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
    const int32_t r = check_grad(h->cfg, i, h->numel[i], grads[i], &h->err);
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
    s.lr = (float)lr;
    s.step = (float)(lr / (1.0 - std::pow(c.beta1, (double)t)));
    s.root2 = (float)(1.0 / std::sqrt(1.0 - std::pow(c.beta2, (double)t)));
    s.eps = (float)c.eps;
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, block, 0, st, s); };
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
