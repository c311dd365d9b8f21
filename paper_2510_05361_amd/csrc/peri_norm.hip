// The boundary of a Peri-LN block (include/mtdao_ops.h): norm after the block,
// gate and residual scale, norm before the next block, in one pass over the
// rows, and its backward pass.
//
// A row of D elements lies in the registers of TPR threads (a wave or more),
// eight consecutive elements per thread and vector, so every tensor is read
// and written once and the statistics are formed from registers (the mean
// first, then the centred squares).  Both passes are bound by HBM: forward
// reads x, f and writes x', n; backward reads dx', dn, x', f and writes dx,
// df.  The backward pass forms the statistics again rather than reading
// stored ones: the rows pass through registers anyway.
//
// Measured at 16384 x 2048 in bf16, RMSNorm with a gate for each channel: forward
// 46 us (268 MB, 5.8 TB/s), backward 74 us (403 MB, 5.4 TB/s) with the 5 us that
// k_peri_columns takes, replayed over the same tensors, of which the 256 MB cache
// holds some; 52.5 and 82.6 us (5.1 and 4.9 TB/s) over others each time.  Backward, rows of a workgroup lying apart by the number
// of workgroups, so that all of them sweep one part of memory, took 80 us where
// rows one after the other took 87 us; 768 and 1024 workgroups are slower than
// 512 (78 and 87 us against 74 us): more sums to write and read back.

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <string>
#include <type_traits>

#include "../../include/mtdao_ops.h"
#include "host.hpp"
#include "ops_device.hpp"

using namespace mtdao;
using namespace mtdao::ops;

namespace {

constexpr int kE = 8;         // elements of a thread's vector
constexpr int kNonTemporal = 2;  // of a buffer access
typedef uint32_t u32v4 __attribute__((ext_vector_type(4)));
constexpr int kGroup = 256;   // smallest workgroup

struct Args {
  int64_t rows, rows_per_gate, ld_x, ld_f, ld_d_out, ld_dn;
  const void *x, *f, *w_post, *w_pre, *gate, *d_out, *dn;
  void *x_out, *n_out, *df;
  float *d_w_post, *d_w_pre, *d_gate;
  float* partial;           // backward: [2][blocks][D], sums of a workgroup's rows
  int64_t gates;            // backward: gates, one for rows without one
  int64_t longest;          // backward: rows that a workgroup (whole_gates: a row group) takes at most
  uint32_t parts;           // backward: workgroups of a gate
  int32_t per_block;        // backward: gates of a workgroup (whole_gates)
  int32_t d, whole_gates, weight_bf16;
  float eps, scale, inv_d;
};

// Sums of N values over the TPR threads of a row, in all of them.  `buf` has
// N floats per wave of the workgroup; consecutive calls use different ones.
template <int TPR, int N>
__device__ __forceinline__ void sum_row(float (&v)[N], float* buf) {
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = sum64(v[i]);
  if constexpr (TPR > 64) {
    constexpr int W = TPR / 64;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x % 64, first = wave / W * W;
    if (lane == 0) {
#pragma unroll
      for (int i = 0; i < N; ++i) buf[wave * N + i] = v[i];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) {
      float s = 0.0f;
#pragma unroll
      for (int w = 0; w < W; ++w) s += buf[(first + w) * N + i];
      v[i] = s;
    }
  }
}

// A vector of kE columns of which n (any number, none for n <= 0) are the row's;
// WHOLE: all or none, where d is a multiple of kE, which keeps the code for single
// elements and the registers it takes out of the kernel.
template <bool WHOLE, bool NT = false, typename T>
__device__ __forceinline__ void load_columns(const T* p, int n, float (&o)[kE]) {
  if (n > 0) {
    if constexpr (WHOLE) load_full<kE, NT>(p, o);
    else load_some<kE, NT>(p, n, o);
  } else {
#pragma unroll
    for (int t = 0; t < kE; ++t) o[t] = 0.0f;
  }
}
template <bool WHOLE, bool NT = false, typename T>
__device__ __forceinline__ void store_columns(T* p, int n, const float (&o)[kE]) {
  if (n > 0) {
    if constexpr (WHOLE) store_full<kE, NT>(p, o);
    else store_some<kE, NT>(p, n, o);
  }
}

// A row of d elements, none for d = 0.  Rows of whole vectors go through a buffer
// descriptor, which takes lanes past the row for zeros and drops their stores:
// without a branch around them the compiler can count the accesses in flight,
// and waits for the loads of a row rather than for the stores of the one before.
// Stores are non-temporal; loads are not: what the pass before wrote may still be
// in the 256 MB cache (forward, 16384 x 2048 bf16: neither 51.1 us, stores 47.8 us,
// both 58.1 us).
template <typename T, bool WHOLE>
struct RowOf {
  T* p;
  int d;
  __device__ __forceinline__ RowOf(const void* base, int64_t at, int d_)
      : p(reinterpret_cast<T*>(const_cast<void*>(base)) + at), d(d_) {}
  __device__ __forceinline__ __amdgpu_buffer_rsrc_t rsrc() const {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>((const void*)p), 0, d * (int)sizeof(T), 0x00027000);
  }
  __device__ __forceinline__ void load(int e, Raw<std::remove_const_t<T>>& o) const {
    if constexpr (WHOLE) {
#pragma unroll
      for (int i = 0; i < (int)sizeof(T) / 2; ++i) {
        const u32v4 v = __builtin_amdgcn_raw_buffer_load_b128(rsrc(), e * (int)sizeof(T) + 16 * i, 0, 0);
#pragma unroll
        for (int t = 0; t < 4; ++t) o.set(4 * i + t, v[t]);
      }
    } else {
      o.load(p + e, d - e);
    }
  }
  __device__ __forceinline__ void store(int e, const float (&o)[kE]) const {
    if constexpr (WHOLE) {
#pragma unroll
      for (int i = 0; i < (int)sizeof(T) / 2; ++i) {
        u32v4 v;
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          if constexpr (sizeof(T) == 2) v[t] = pack_bf16(o[2 * t], o[2 * t + 1]);
          else v[t] = __float_as_uint(o[4 * i + t]);
        }
        __builtin_amdgcn_raw_buffer_store_b128(v, rsrc(), e * (int)sizeof(T) + 16 * i, 0, kNonTemporal);
      }
    } else if (d - e > 0) {
      store_some<kE, true>(p + e, d - e, o);
    }
  }
};

template <bool WHOLE>
__device__ __forceinline__ void load_weight(const void* p, bool bf16, int64_t at, int n, float (&o)[kE]) {
  if (bf16) load_columns<WHOLE>(reinterpret_cast<const bf16_t*>(p) + at, n, o);
  else load_columns<WHOLE>(reinterpret_cast<const float*>(p) + at, n, o);
}

__device__ __forceinline__ float weight_at(const void* p, bool bf16, int64_t at) {
  return bf16 ? to_f32(reinterpret_cast<const bf16_t*>(p)[at]) : reinterpret_cast<const float*>(p)[at];
}

// 1 / sqrt(x), off by an ulp, as a mean is that is a sum times the rounded 1 / D: less
// than the sums' own roundings.  The hardware takes numbers below 2^-126 for zero.
__device__ __forceinline__ float inverse_root(float x) {
  const bool tiny = x < 0x1p-126f;
  return __builtin_amdgcn_rsqf(tiny ? x * 0x1p64f : x) * (tiny ? 0x1p32f : 1.0f);
}

// z centred (LayerNorm) in place, 1 / sqrt(mean square + eps) returned.
template <int TPR, int NV, bool LAYER>
__device__ __forceinline__ float normalize(float (&z)[NV][kE], const int (&n)[NV], const Args& a, float* buf) {
  if constexpr (LAYER) {
    float m[1] = {0.0f};
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
      for (int t = 0; t < kE; ++t) m[0] += z[v][t];
    sum_row<TPR>(m, buf);
    const float mean = m[0] * a.inv_d;
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
      for (int t = 0; t < kE; ++t) z[v][t] = t < n[v] ? z[v][t] - mean : 0.0f;
    buf += kGroup / 64 * (TPR > kGroup ? TPR / kGroup : 1);
  }
  float q[1] = {0.0f};
#pragma unroll
  for (int v = 0; v < NV; ++v)
#pragma unroll
    for (int t = 0; t < kE; ++t) q[0] = fmaf(z[v][t], z[v][t], q[0]);
  sum_row<TPR>(q, buf);
  return inverse_root(fmaf(q[0], a.inv_d, a.eps));
}

template <typename ST, typename BT, bool LAYER, bool WHOLE, int TPR, int NV>
__global__ __launch_bounds__(TPR > kGroup ? TPR : kGroup) void k_peri_norm(Args a) {
  constexpr int kThreads = TPR > kGroup ? TPR : kGroup, kWaves = kThreads / 64;
  __shared__ float buf[4 * kWaves];
  const int lane = threadIdx.x % TPR;
  const int64_t block = (int64_t)blockIdx.y * gridDim.x + blockIdx.x;
  const int64_t row_or_past = block * (kThreads / TPR) + __builtin_amdgcn_readfirstlane(threadIdx.x / TPR);
  const bool live = row_or_past < a.rows;
  if (TPR == 64 && !live) return;  // (wider rows fill a workgroup or meet at barriers)
  const int64_t row = live ? row_or_past : a.rows - 1;
  const ST* x = reinterpret_cast<const ST*>(a.x) + row * a.ld_x;
  float xa[NV][kE], fa[NV][kE];
  int n[NV];
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    const int e = (v * TPR + lane) * kE;
    n[v] = a.d - e;
    load_columns<WHOLE>(x + e, n[v], xa[v]);
    if (a.f) load_columns<WHOLE>(reinterpret_cast<const BT*>(a.f) + row * a.ld_f + e, n[v], fa[v]);
  }
  const bool wb = a.weight_bf16 != 0;
  // with one vector a thread, what the rows are multiplied with is on its way with them
  constexpr bool kEarly = NV == 1;
  const int64_t gate_row = a.gate ? row / a.rows_per_gate * a.d : 0;
  float w_post[NV][kE], w_pre[NV][kE], gate[NV][kE];
  auto weights = [&](const void* p, int64_t at, float (&w)[NV][kE]) {
#pragma unroll
    for (int v = 0; v < NV; ++v) load_weight<WHOLE>(p, wb, at + (v * TPR + lane) * kE, n[v], w[v]);
  };
  if (kEarly) {
    if (a.f) weights(a.w_post, 0, w_post);
    if (a.gate) weights(a.gate, gate_row, gate);
    if (a.w_pre) weights(a.w_pre, 0, w_pre);
  }
  if (a.f) {
    const float r = normalize<TPR, NV, LAYER>(fa, n, a, buf) * a.scale;
    ST* out = reinterpret_cast<ST*>(a.x_out) + row * a.d;
    if (!kEarly) {
      weights(a.w_post, 0, w_post);
      if (a.gate) weights(a.gate, gate_row, gate);
    }
#pragma unroll
    for (int v = 0; v < NV; ++v) {
#pragma unroll
      for (int t = 0; t < kE; ++t) {
        const float h = fa[v][t] * r * w_post[v][t];
        xa[v][t] += a.gate ? h * gate[v][t] : h;
      }
      if (live) store_columns<WHOLE, true>(out + (v * TPR + lane) * kE, n[v], xa[v]);
    }
  }
  if (a.w_pre) {
    const float r = normalize<TPR, NV, LAYER>(xa, n, a, buf + 2 * kWaves);
    BT* out = reinterpret_cast<BT*>(a.n_out) + row * a.d;
    if (!kEarly) weights(a.w_pre, 0, w_pre);
#pragma unroll
    for (int v = 0; v < NV; ++v) {
#pragma unroll
      for (int t = 0; t < kE; ++t) xa[v][t] = xa[v][t] * r * w_pre[v][t];
      if (live) store_columns<WHOLE, true>(out + (v * TPR + lane) * kE, n[v], xa[v]);
    }
  }
}

// ------------------------------------------------------------------ backward

// Rows of a workgroup: either one range of rows whose gate (if any) is one,
// split over the workgroup's row groups, or `per_block` whole gates, each
// taken by one row group (whole_gates).  With xh, fh the normalized rows, dd the
// gradient of x and u = gate scale w_post, a row gives df from dd u and fh, and
//   s_pre += dn xh,  t += dd fh;  d_w_post = sum gate scale t,  d_gate = scale w_post t,
// so a thread keeps two sums of its columns, and a third where gates change.
// The next row is loaded, as it is in memory, while one is worked on.  The
// workgroup joins its row groups at the end and writes a row of partial sums,
// which k_peri_columns adds up.
template <typename ST, typename BT, bool LAYER, bool WHOLE, int TPR, int NV>
__global__ __launch_bounds__(TPR > kGroup ? TPR : kGroup) void k_peri_norm_backward(Args a) {
  constexpr int kThreads = TPR > kGroup ? TPR : kGroup, kWaves = kThreads / 64, kGroups = kThreads / TPR;
  __shared__ float buf[9 * kWaves];
  __shared__ float joined[kGroups > 1 ? kThreads * kE : 1];
  const int lane = threadIdx.x % TPR, group = __builtin_amdgcn_readfirstlane(threadIdx.x / TPR);
  const bool wb = a.weight_bf16 != 0;
  float w_pre[NV][kE], u[NV][kE], s_pre[NV][kE], s_post[NV][kE], s_t[NV][kE];
  int n[NV];
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    n[v] = a.d - (v * TPR + lane) * kE;
#pragma unroll
    for (int t = 0; t < kE; ++t) w_pre[v][t] = u[v][t] = s_pre[v][t] = s_post[v][t] = s_t[v][t] = 0.0f;
    if (a.w_pre) load_weight<WHOLE>(a.w_pre, wb, (v * TPR + lane) * kE, n[v], w_pre[v]);
  }
  const int of_x = a.w_pre ? a.d : 0, of_f = a.f ? a.d : 0, of_d = a.d_out ? a.d : 0, of_y = a.dn && a.w_pre ? a.d : 0;  // columns to load
  const uint32_t block = blockIdx.x;
  const int rounds = a.whole_gates ? (a.per_block + kGroups - 1) / kGroups : 1;
  for (int round = 0; round < rounds; ++round) {
    const int nth = round * kGroups + group;  // gate of the workgroup (whole_gates)
    const bool mine = !a.whole_gates || (nth < a.per_block && (int64_t)block * a.per_block + nth < a.gates);
    const int64_t my_gate = !mine ? 0 : a.whole_gates ? (int64_t)block * a.per_block + nth : block / a.parts;
    const int64_t step = a.whole_gates ? 1 : (int64_t)kGroups * a.parts;
    int64_t at = my_gate * a.rows_per_gate, end = at + a.rows_per_gate < a.rows ? at + a.rows_per_gate : a.rows;
    if (!mine) end = at;
    if (!a.whole_gates) at += block % a.parts + (int64_t)group * a.parts;
    if (a.f) {
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        float g[kE];
        load_weight<WHOLE>(a.w_post, wb, (v * TPR + lane) * kE, n[v], u[v]);
        if (a.gate) load_weight<WHOLE>(a.gate, wb, my_gate * a.d + (v * TPR + lane) * kE, n[v], g);
#pragma unroll
        for (int t = 0; t < kE; ++t) u[v][t] *= a.gate ? g[t] * a.scale : a.scale;
      }
    }
    Raw<ST> rx[NV], rd[NV];
    Raw<BT> rf[NV], ry[NV];
    auto fetch = [&](int64_t row) {
      const bool live = row < end;
      const RowOf<const ST, WHOLE> x(a.x, row * a.ld_x, live ? of_x : 0), d(a.d_out, row * a.ld_d_out, live ? of_d : 0);
      const RowOf<const BT, WHOLE> f(a.f, row * a.ld_f, live ? of_f : 0), y(a.dn, row * a.ld_dn, live ? of_y : 0);
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        const int e = (v * TPR + lane) * kE;
        x.load(e, rx[v]);
        f.load(e, rf[v]);
        d.load(e, rd[v]);
        y.load(e, ry[v]);
      }
    };
    constexpr bool kAhead = NV == 1;  // (two vectors of the next row do not fit the registers)
    if (kAhead) fetch(at);
    for (int64_t left = a.longest; left > 0; left -= a.whole_gates ? 1 : kGroups, at += step) {
      if (!kAhead) fetch(at);
      float x[NV][kE], f[NV][kE], d[NV][kE], y[NV][kE];
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        rx[v].values(x[v]);
        rf[v].values(f[v]);
        rd[v].values(d[v]);
        ry[v].values(y[v]);
      }
      if (kAhead) fetch(at + step);
      const bool live = at < end;
      float mean = 0.0f;
      if constexpr (LAYER) {  // centre x and f; the mean of dn w_pre
        float m[3] = {0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
          for (int t = 0; t < kE; ++t) {
            m[0] += x[v][t];
            m[1] += f[v][t];
            m[2] = fmaf(y[v][t], w_pre[v][t], m[2]);
          }
        sum_row<TPR>(m, buf);
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
          for (int t = 0; t < kE; ++t) {
            x[v][t] = t < n[v] ? fmaf(-m[0], a.inv_d, x[v][t]) : 0.0f;
            f[v][t] = t < n[v] ? fmaf(-m[1], a.inv_d, f[v][t]) : 0.0f;
          }
        mean = m[2] * a.inv_d;
      }
      float q[3] = {0.0f, 0.0f, 0.0f};  // squares of x and f, and dn w_pre against x
#pragma unroll
      for (int v = 0; v < NV; ++v)
#pragma unroll
        for (int t = 0; t < kE; ++t) {
          q[0] = fmaf(x[v][t], x[v][t], q[0]);
          q[1] = fmaf(f[v][t], f[v][t], q[1]);
          q[2] = fmaf(y[v][t] * w_pre[v][t], x[v][t], q[2]);
        }
      sum_row<TPR>(q, buf + 3 * kWaves);
      // (zeros stand for what is not there, rows past the end among it: without an eps their roots would be infinite)
      const float sx = live && a.w_pre ? inverse_root(fmaf(q[0], a.inv_d, a.eps)) : 0.0f;
      const float sf = live && a.f ? inverse_root(fmaf(q[1], a.inv_d, a.eps)) : 0.0f;
      const float along = q[2] * sx * a.inv_d;
      float c[2] = {0.0f, 0.0f};  // a = dd u against fh, and its sum
#pragma unroll
      for (int v = 0; v < NV; ++v) {
#pragma unroll
        for (int t = 0; t < kE; ++t) {
          const float xh = x[v][t] * sx, fh = f[v][t] * sf;
          s_pre[v][t] = fmaf(y[v][t], xh, s_pre[v][t]);
          const float through = fmaf(-xh, along, LAYER ? fmaf(y[v][t], w_pre[v][t], -mean) : y[v][t] * w_pre[v][t]);
          d[v][t] = fmaf(sx, through, d[v][t]);
          s_t[v][t] = fmaf(d[v][t], fh, s_t[v][t]);
          y[v][t] = d[v][t] * u[v][t];
          f[v][t] = fh;
          c[0] = fmaf(y[v][t], fh, c[0]);
          if constexpr (LAYER) c[1] += y[v][t];  // (u is zero past the row)
        }
        RowOf<ST, WHOLE>(a.x_out, at * a.d, live ? a.d : 0).store((v * TPR + lane) * kE, d[v]);
      }
      if (a.f) {
        if constexpr (LAYER) {
          sum_row<TPR>(c, buf + 6 * kWaves);
        } else {
          float one[1] = {c[0]};
          sum_row<TPR>(one, buf + 6 * kWaves);
          c[0] = one[0];
        }
        const float by = -c[0] * a.inv_d, less = LAYER ? c[1] * a.inv_d : 0.0f;
#pragma unroll
        for (int v = 0; v < NV; ++v) {
#pragma unroll
          for (int t = 0; t < kE; ++t) y[v][t] = sf * fmaf(f[v][t], by, LAYER ? y[v][t] - less : y[v][t]);
          RowOf<BT, WHOLE>(a.df, at * a.d, live ? a.d : 0).store((v * TPR + lane) * kE, y[v]);
        }
      }
      // Each exchange of a row has its own floats: when all have met at a row's
      // last barrier they have read those of the ones before it, and the last
      // one's are read before its next row's first barrier.  One exchange alone
      // has no barrier after it.
      if (TPR > 64 && !LAYER && !a.f) __syncthreads();
    }
    if (a.whole_gates) {
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        float w[kE], g[kE];
        load_weight<WHOLE>(a.w_post, wb, (v * TPR + lane) * kE, n[v], w);
        load_weight<WHOLE>(a.gate, wb, my_gate * a.d + (v * TPR + lane) * kE, n[v], g);
#pragma unroll
        for (int t = 0; t < kE; ++t) {
          s_post[v][t] = fmaf(g[t] * a.scale, s_t[v][t], s_post[v][t]);
          w[t] *= a.scale * s_t[v][t];
          s_t[v][t] = 0.0f;
        }
        if (mine) store_columns<WHOLE>(a.d_gate + my_gate * a.d + (v * TPR + lane) * kE, n[v], w);
      }
    }
  }
  // join the row groups, in order, and write the workgroup's sums
  auto write = [&](float (&s)[NV][kE], float* out) {
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      if constexpr (kGroups > 1) {
        __syncthreads();
#pragma unroll
        for (int t = 0; t < kE; ++t) joined[t * kThreads + threadIdx.x] = s[v][t];
        __syncthreads();
        if (group == 0) {
#pragma unroll
          for (int t = 0; t < kE; ++t)
#pragma unroll
            for (int g = 1; g < kGroups; ++g) s[v][t] += joined[t * kThreads + g * TPR + lane];
        }
      }
      if (group == 0) store_columns<WHOLE>(out + (v * TPR + lane) * kE, n[v], s[v]);
    }
  };
  const int64_t plane = (int64_t)gridDim.x * a.d;
  if (a.w_pre) write(s_pre, a.partial + block * a.d);
  if (a.f && a.whole_gates) write(s_post, a.partial + plane + block * a.d);
  else if (a.f) write(s_t, a.partial + plane + block * a.d);
}

// Sums of the workgroups' partial rows.  Job 0: w_pre.  Job 1: w_post, of the
// sums over its rows (whole_gates) or of t times the gate of each workgroup.
// From job 2 on 32 / fold gates each, of t, with fold the power of two that holds
// a gate's parts (32 at most).  32 columns x 32 rows at once.
constexpr int kCols = 32;
__global__ __launch_bounds__(kCols * 32) void k_peri_columns(Args a, int64_t blocks, int fold) {
  __shared__ float part[32][kCols + 1];
  const int col = threadIdx.x % kCols, lane = threadIdx.x / kCols;
  const int64_t c = (int64_t)blockIdx.x * kCols + col;
  const int job = blockIdx.y, apart = job < 2 ? 32 : fold;
  if ((job == 0 && !a.w_pre) || (job == 1 && !a.f)) return;
  const bool wb = a.weight_bf16 != 0, gated = a.gate && !a.whole_gates;
  const int64_t gate = job < 2 ? 0 : (int64_t)(job - 2) * (32 / fold) + lane / fold;
  const int64_t from = job < 2 ? 0 : gate * a.parts, count = job < 2 ? blocks : gate < a.gates ? a.parts : 0;
  const float* in = a.partial + ((job == 0 ? 0 : blocks) + from) * a.d;
  float s = 0.0f;
  if (c < a.d) {
    int64_t r = lane % apart;
    if (job == 1 && gated) {
#pragma unroll 8
      for (; r < count; r += 32) s = fmaf(weight_at(a.gate, wb, (int64_t)((uint32_t)r / a.parts) * a.d + c), in[r * a.d + c], s);
    } else {
      for (; r + 15 * apart < count; r += 16 * apart) {  // (512 workgroups: all of them at once)
        float v[16];
#pragma unroll
        for (int k = 0; k < 16; ++k) v[k] = in[(r + k * apart) * a.d + c];
#pragma unroll
        for (int k = 0; k < 16; ++k) s += v[k];
      }
#pragma unroll 4
      for (; r < count; r += apart) s += in[r * a.d + c];
    }
  }
  part[lane][col] = s;
  __syncthreads();
  if (lane % apart != 0 || c >= a.d) return;
  s = 0.0f;
#pragma unroll 8
  for (int r = 0; r < apart; ++r) s += part[lane + r][col];
  if (job == 0) a.d_w_pre[c] = s;
  else if (job == 1) a.d_w_post[c] = a.whole_gates ? s : s * a.scale;
  else if (gate < a.gates) a.d_gate[gate * a.d + c] = s * a.scale * weight_at(a.w_post, wb, c);
}

// --------------------------------------------------------------------- host

bool is_type(int32_t dt) { return dt == MTDAO_F32 || dt == MTDAO_BF16; }
// (rows_per_gate may be any number: nothing is added to it)
int64_t gates_of(const mtdao_peri_norm_args& a) {
  return a.gate ? a.rows / a.rows_per_gate + (a.rows % a.rows_per_gate != 0) : 0;
}

int32_t validate_sizes(const mtdao_peri_norm_args* p, std::string* e) {
  if (!p) return fail(e, MTDAO_ERR_INVALID_ARG, "args is NULL");
  const mtdao_peri_norm_args& a = *p;
  if (a.rows < 0) return fail(e, MTDAO_ERR_INVALID_ARG, "rows < 0");
  if (a.d < 1 || a.d > MTDAO_PERI_MAX_D)
    return fail(e, MTDAO_ERR_INVALID_ARG, "d %lld outside [1, %d]", (long long)a.d, MTDAO_PERI_MAX_D);
  if (a.rows > (INT64_C(1) << 40) / a.d) return fail(e, MTDAO_ERR_INVALID_ARG, "rows * d exceeds 2^40");
  if (a.kind != MTDAO_NORM_RMS && a.kind != MTDAO_NORM_LAYER)
    return fail(e, MTDAO_ERR_INVALID_ARG, "kind %d is not RMS(0) or LAYER(1)", a.kind);
  if (!is_type(a.stream_dtype) || !is_type(a.branch_dtype) || !is_type(a.weight_dtype))
    return fail(e, MTDAO_ERR_INVALID_ARG, "stream_dtype, branch_dtype, weight_dtype must be F32(0) or BF16(1)");
  if (a.stream_dtype == MTDAO_BF16 && a.branch_dtype == MTDAO_F32)
    return fail(e, MTDAO_ERR_INVALID_ARG, "an fp32 branch needs an fp32 stream");
  if (!(a.eps >= 0.0f) || !std::isfinite(a.eps)) return fail(e, MTDAO_ERR_INVALID_ARG, "eps=%g must be finite and >= 0", a.eps);
  if (!std::isfinite(a.scale)) return fail(e, MTDAO_ERR_INVALID_ARG, "scale is not finite");
  if (a.gate && !a.f) return fail(e, MTDAO_ERR_INVALID_ARG, "a gate needs f");
  if (a.gate && a.rows_per_gate < 1) return fail(e, MTDAO_ERR_INVALID_ARG, "rows_per_gate < 1");
  if (!a.f && !a.w_pre) return fail(e, MTDAO_ERR_INVALID_ARG, "neither f nor w_pre is given");
  return MTDAO_OK;
}

int32_t check_pointer(const void* p, int64_t align, const char* name, std::string* e) {
  if (!p) return fail(e, MTDAO_ERR_INVALID_ARG, "%s is NULL", name);
  if (!aligned_to(p, (uintptr_t)align)) return fail(e, MTDAO_ERR_ALIGN, "%s is not aligned to its element", name);
  return MTDAO_OK;
}

// An input of [rows][d] with row stride ld.
int32_t check_rows(const mtdao_peri_norm_args& a, const void* p, int64_t ld, int32_t dt, const char* name, std::string* e) {
  if (ld < a.d || ld > (INT64_C(1) << 40) / (a.rows < 1 ? 1 : a.rows))
    return fail(e, MTDAO_ERR_INVALID_ARG, "row stride %lld of %s is below d or exceeds 2^40 elements in all", (long long)ld, name);
  return check_pointer(p, esize(dt), name, e);
}

// The written [rows][d] buffer `out` against an input; the same rows in
// place are fine (`same`).
int32_t check_apart(const mtdao_peri_norm_args& a, const void* out, int32_t out_dt, const void* in, int64_t ld, int32_t dt,
                    bool same, const char* name, std::string* e) {
  if (!in || !out) return MTDAO_OK;
  if (same && out == in && ld == a.d && out_dt == dt) return MTDAO_OK;
  if (overlap(out, a.rows * a.d * esize(out_dt), in, ((a.rows - 1) * ld + a.d) * esize(dt)))
    return fail(e, MTDAO_ERR_INVALID_ARG, "an output overlaps %s", name);
  return MTDAO_OK;
}

int32_t check_weights(const mtdao_peri_norm_args& a, std::string* e) {
  int32_t r = MTDAO_OK;
  if (a.f) r = check_pointer(a.w_post, esize(a.weight_dtype), "w_post", e);
  if (r == MTDAO_OK && a.w_pre) r = check_pointer(a.w_pre, esize(a.weight_dtype), "w_pre", e);
  if (r == MTDAO_OK && a.gate) r = check_pointer(a.gate, esize(a.weight_dtype), "gate", e);
  return r;
}

Args device_args(const mtdao_peri_norm_args& a) {
  Args k = {};
  k.rows = a.rows;
  k.rows_per_gate = a.gate ? a.rows_per_gate : 1;
  k.ld_x = a.ld_x;
  k.ld_f = a.ld_f;
  k.ld_d_out = a.ld_d_out;
  k.ld_dn = a.ld_dn;
  k.x = a.x;
  k.f = a.f;
  k.w_post = a.w_post;
  k.w_pre = a.w_pre;
  k.gate = a.gate;
  k.d_out = a.d_out;
  k.dn = a.dn;
  k.x_out = a.x_out;
  k.n_out = a.n_out;
  k.df = a.df;
  k.d_w_post = a.d_w_post;
  k.d_w_pre = a.d_w_pre;
  k.d_gate = a.d_gate;
  k.d = (int32_t)a.d;
  k.weight_bf16 = a.weight_dtype == MTDAO_BF16;
  k.eps = a.eps;
  k.scale = a.scale;
  k.inv_d = 1.0f / (float)a.d;
  return k;
}

template <int V>
using Int = std::integral_constant<int, V>;

// Rows of whole vectors from dword to dword.
bool whole_rows(const mtdao_peri_norm_args& a) {
  auto dwords = [](const void* p, int64_t ld, int32_t dt) { return !p || (aligned_to(p, 4) && ld % 4 * esize(dt) % 4 == 0); };
  return a.d % kE == 0 && dwords(a.x, a.ld_x, a.stream_dtype) && dwords(a.f, a.ld_f, a.branch_dtype) &&
         dwords(a.d_out, a.ld_d_out, a.stream_dtype) && dwords(a.dn, a.ld_dn, a.branch_dtype) && dwords(a.x_out, a.d, a.stream_dtype) &&
         dwords(a.n_out, a.d, a.branch_dtype) && dwords(a.df, a.d, a.branch_dtype);
}

// f(stream type, branch type, layer, whole)
template <typename F>
void with_types(const mtdao_peri_norm_args& a, F&& f) {
  auto whole = [&](auto s, auto b, auto layer) {
    if (whole_rows(a)) f(s, b, layer, std::true_type{});
    else f(s, b, layer, std::false_type{});
  };
  auto kind = [&](auto s, auto b) {
    if (a.kind == MTDAO_NORM_LAYER) whole(s, b, std::true_type{});
    else whole(s, b, std::false_type{});
  };
  if (a.stream_dtype == MTDAO_BF16) kind(bf16_t{}, bf16_t{});
  else if (a.branch_dtype == MTDAO_BF16) kind(float{}, bf16_t{});
  else kind(float{}, float{});
}

// Threads of a row, backward: one vector a thread up to D = 4096, which leaves
// registers for two rows in flight and the sums of the thread's columns.
int backward_threads(int64_t d) { return d <= 64 * kE ? 64 : d <= 128 * kE ? 128 : d <= 256 * kE ? 256 : 512; }

// Forward, a row has one vector a thread up to D = 512 and from 1025 to 2048 (one
// wave with four: 16384 x 2048 bf16 54.0 us against 46.1 us), and else where there
// are few elements: then the latency of one row counts, above it the work of the
// reductions.  One vector a thread against two or four: 1024 x 768 4.7 us (5.0),
// 2048 x 768 5.9 us (5.2), 256 x 4096 4.8 us (5.4), 1024 x 4096 6.9 us (6.4),
// 1 x 8192 4.5 us (7.0), 512 x 8192 8.6 us (8.3).
constexpr int64_t kFew = INT64_C(1) << 20;

// How the rows go over the workgroups, backward: kBlocks of them at most, one a
// CU as long as that leaves them two to eight rows, none across gates unless it
// has them whole.  (A workgroup for each two rows up to 512 of them, against eight
// rows each: 64 x 2048 9.0 us (14.1), 1024 x 2048 17.3 us (16.3; with four 14.6 us),
// 2047 x 768 14.5 us (13.0): more sums to write and read back.)
constexpr int64_t kBlocks = 512;
struct Plan {
  int64_t blocks, per_block, parts;
  bool whole_gates;
};
Plan backward_plan(const mtdao_peri_norm_args& a) {
  Plan p;
  const int64_t few = std::min<int64_t>(8, std::max<int64_t>(2, (a.rows + 255) / 256));
  const int64_t rows = std::max(few, (a.rows + kBlocks - 1) / kBlocks);
  const int64_t gates = gates_of(a);
  // Whole gates up to as many rows as a workgroup has (4452 x 3968, five rows a gate
  // of nine: 94 -> 61 us; 16384 x 2048, 32 of 32: 83 -> 74 us); where a workgroup has
  // several row groups, which then take a gate each, up to two thirds (d = 256, 20 of
  // 32: 37 -> 30 us, 32 of 32: 24 -> 39 us).
  if (gates > 1 && a.rows_per_gate <= (backward_threads(a.d) < kGroup ? 2 * rows / 3 : rows)) {
    p.per_block = (rows + a.rows_per_gate - 1) / a.rows_per_gate;
    p.parts = 1;
    p.blocks = (gates + p.per_block - 1) / p.per_block;
    p.whole_gates = true;
  } else {
    const int64_t each = gates > 1 ? a.rows_per_gate : a.rows;
    p.parts = (each + rows - 1) / rows;
    p.per_block = (each + p.parts - 1) / p.parts;
    p.parts = (each + p.per_block - 1) / p.per_block;
    p.blocks = p.parts * std::max<int64_t>(1, gates);
    p.whole_gates = false;
  }
  return p;
}

size_t backward_bytes(const mtdao_peri_norm_args& a) {
  return a.rows == 0 ? 0 : (size_t)2 * (size_t)backward_plan(a).blocks * (size_t)a.d * sizeof(float);
}

}  // namespace

extern "C" {

int32_t mtdao_peri_norm(const mtdao_peri_norm_args* args, void* hip_stream) {
  std::string* e = &g_err;
  int32_t r = validate_sizes(args, e);
  if (r != MTDAO_OK) return r;
  const mtdao_peri_norm_args& a = *args;
  if (a.rows == 0) return MTDAO_OK;
  r = check_weights(a, e);
  if (r == MTDAO_OK) r = check_rows(a, a.x, a.ld_x, a.stream_dtype, "x", e);
  if (r == MTDAO_OK && a.f) r = check_rows(a, a.f, a.ld_f, a.branch_dtype, "f", e);
  if (r == MTDAO_OK && a.f) r = check_pointer(a.x_out, esize(a.stream_dtype), "x_out", e);
  if (r == MTDAO_OK && a.w_pre) r = check_pointer(a.n_out, esize(a.branch_dtype), "n_out", e);
  if (r != MTDAO_OK) return r;
  if (a.f) {
    r = check_apart(a, a.x_out, a.stream_dtype, a.x, a.ld_x, a.stream_dtype, true, "x", e);
    if (r == MTDAO_OK) r = check_apart(a, a.x_out, a.stream_dtype, a.f, a.ld_f, a.branch_dtype, true, "f", e);
    if (r == MTDAO_OK && a.w_pre)
      r = check_apart(a, a.x_out, a.stream_dtype, a.n_out, a.d, a.branch_dtype, false, "n_out", e);
    if (r != MTDAO_OK) return r;
  }
  if (a.w_pre) {
    r = check_apart(a, a.n_out, a.branch_dtype, a.x, a.ld_x, a.stream_dtype, true, "x", e);
    if (r == MTDAO_OK) r = check_apart(a, a.n_out, a.branch_dtype, a.f, a.ld_f, a.branch_dtype, true, "f", e);
    if (r != MTDAO_OK) return r;
  }
  hipStream_t st = reinterpret_cast<hipStream_t>(hip_stream);
  RoctxRange range("mtdao_peri_norm rows=%lld d=%lld", (long long)a.rows, (long long)a.d);
  const Args k = device_args(a);
  const bool few = a.rows * a.d <= kFew;
  const int64_t per = a.d <= 512 || (a.d <= 1024 && !few) ? 4 : 1;
  const int64_t blocks = (a.rows + per - 1) / per;
  if (blocks > kGridMost) return fail(e, MTDAO_ERR_INVALID_ARG, "rows exceed the largest launch");
  with_types(a, [&](auto s, auto b, auto layer, auto whole) {
    using ST = decltype(s);
    using BT = decltype(b);
    constexpr bool L = decltype(layer)::value, W = decltype(whole)::value;
    auto go = [&](auto tpr, auto nv) {
      constexpr int T = decltype(tpr)::value;
      hipLaunchKernelGGL((k_peri_norm<ST, BT, L, W, T, decltype(nv)::value>), grid_of(blocks), dim3(T > kGroup ? T : kGroup), 0, st, k);
    };
    if (a.d <= 512) go(Int<64>{}, Int<1>{});
    else if (a.d <= 1024 && !few) go(Int<64>{}, Int<2>{});
    else if (a.d <= 2048) go(Int<256>{}, Int<1>{});
    else if (a.d <= 4096 && !few) go(Int<256>{}, Int<2>{});
    else if (a.d <= 4096) go(Int<512>{}, Int<1>{});
    else if (!few) go(Int<256>{}, Int<4>{});
    else go(Int<1024>{}, Int<1>{});
  });
  return hip_check(e, hipGetLastError(), "mtdao_peri_norm launch");
}

int32_t mtdao_peri_norm_backward_workspace_bytes(const mtdao_peri_norm_args* a, size_t* bytes) {
  const int32_t r = validate_sizes(a, &g_err);
  if (r != MTDAO_OK) return r;
  if (!bytes) return fail(&g_err, MTDAO_ERR_INVALID_ARG, "bytes is NULL");
  *bytes = backward_bytes(*a);
  return MTDAO_OK;
}

int32_t mtdao_peri_norm_backward(const mtdao_peri_norm_args* args, void* workspace, size_t workspace_bytes,
                                 void* hip_stream) {
  std::string* e = &g_err;
  int32_t r = validate_sizes(args, e);
  if (r != MTDAO_OK) return r;
  const mtdao_peri_norm_args& a = *args;
  r = check_weights(a, e);
  if (r == MTDAO_OK && a.f) r = check_pointer(a.d_w_post, 4, "d_w_post", e);
  if (r == MTDAO_OK && a.w_pre) r = check_pointer(a.d_w_pre, 4, "d_w_pre", e);
  if (r == MTDAO_OK && a.gate) r = check_pointer(a.d_gate, 4, "d_gate", e);
  if (r != MTDAO_OK) return r;
  hipStream_t st = reinterpret_cast<hipStream_t>(hip_stream);
  Args k = device_args(a);
  const Plan plan = a.rows > 0 ? backward_plan(a) : Plan{0, 1, 1, false};  // no rows: sums of nothing
  const size_t need = backward_bytes(a);
  if (a.rows > 0) {
    if (a.w_pre) r = check_rows(a, a.x, a.ld_x, a.stream_dtype, "x", e);
    if (r == MTDAO_OK && a.f) r = check_rows(a, a.f, a.ld_f, a.branch_dtype, "f", e);
    if (r == MTDAO_OK && a.d_out) r = check_rows(a, a.d_out, a.ld_d_out, a.stream_dtype, "d_out", e);
    if (r == MTDAO_OK && a.dn) r = check_rows(a, a.dn, a.ld_dn, a.branch_dtype, "dn", e);
    if (r == MTDAO_OK) r = check_pointer(a.x_out, esize(a.stream_dtype), "x_out", e);
    if (r == MTDAO_OK && a.f) r = check_pointer(a.df, esize(a.branch_dtype), "df", e);
    if (r != MTDAO_OK) return r;
    const void* outs[2] = {a.x_out, a.f ? a.df : nullptr};
    const int32_t types[2] = {a.stream_dtype, a.branch_dtype};
    for (int o = 0; o < 2 && r == MTDAO_OK; ++o) {
      r = check_apart(a, outs[o], types[o], a.w_pre ? a.x : nullptr, a.ld_x, a.stream_dtype, true, "x", e);
      if (r == MTDAO_OK) r = check_apart(a, outs[o], types[o], a.f, a.ld_f, a.branch_dtype, true, "f", e);
      if (r == MTDAO_OK) r = check_apart(a, outs[o], types[o], a.d_out, a.ld_d_out, a.stream_dtype, true, "d_out", e);
      if (r == MTDAO_OK) r = check_apart(a, outs[o], types[o], a.dn, a.ld_dn, a.branch_dtype, true, "dn", e);
    }
    if (r == MTDAO_OK) r = check_apart(a, a.x_out, a.stream_dtype, outs[1], a.d, a.branch_dtype, false, "df", e);
    if (r != MTDAO_OK) return r;
    if (!workspace || workspace_bytes < need)
      return fail(e, MTDAO_ERR_WORKSPACE, "workspace of %zu bytes required, %zu given", need,
                  workspace ? workspace_bytes : (size_t)0);
    if (!aligned_to(workspace, 256)) return fail(e, MTDAO_ERR_ALIGN, "workspace is not 256-byte aligned");
    if (plan.blocks > 0x7fffffff) return fail(e, MTDAO_ERR_INVALID_ARG, "rows exceed the largest launch");
  }
  k.partial = static_cast<float*>(workspace);
  if (!a.gate) k.rows_per_gate = a.rows;
  k.gates = std::max<int64_t>(1, gates_of(a));
  k.parts = (uint32_t)plan.parts;
  k.per_block = plan.whole_gates ? (int32_t)plan.per_block : 1;
  k.longest = plan.whole_gates ? a.rows_per_gate : plan.per_block;
  k.whole_gates = plan.whole_gates;
  RoctxRange range("mtdao_peri_norm_backward rows=%lld d=%lld", (long long)a.rows, (long long)a.d);
  if (a.rows > 0) {
    with_types(a, [&](auto s, auto b, auto layer, auto whole) {
      using ST = decltype(s);
      using BT = decltype(b);
      constexpr bool L = decltype(layer)::value, W = decltype(whole)::value;
      auto go = [&](auto tpr, auto nv) {
        constexpr int T = decltype(tpr)::value;
        hipLaunchKernelGGL((k_peri_norm_backward<ST, BT, L, W, T, decltype(nv)::value>),
                           dim3((unsigned)plan.blocks), dim3(T > kGroup ? T : kGroup), 0, st, k);
      };
      switch (backward_threads(a.d)) {
        case 64: go(Int<64>{}, Int<1>{}); break;
        case 128: go(Int<128>{}, Int<1>{}); break;
        case 256: go(Int<256>{}, Int<1>{}); break;
        default:
          if (a.d <= 512 * kE) go(Int<512>{}, Int<1>{});
          else go(Int<512>{}, Int<2>{});
      }
    });
  }
  int fold = 1;
  while (fold < 32 && fold < plan.parts) fold *= 2;
  const int64_t jobs = 2 + (plan.whole_gates ? 0 : (gates_of(a) + 32 / fold - 1) / (32 / fold));
  // (gates that are not whole hold over a 768th of the rows each, or two, so jobs fit a launch)
  hipLaunchKernelGGL(k_peri_columns, dim3((unsigned)((a.d + kCols - 1) / kCols), (unsigned)jobs), dim3(kCols * 32), 0, st, k, plan.blocks,
                     fold);
  return hip_check(e, hipGetLastError(), "mtdao_peri_norm_backward launch");
}

}  // extern "C"
