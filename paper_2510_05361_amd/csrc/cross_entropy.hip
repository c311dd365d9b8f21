// Cross entropy of rows of logits and its gradient (include/mtdao_ops.h).
//
// For the gradient a row of up to 65536 logits (bf16: 131072) lies in the registers of a wave or a workgroup,
// as it is in memory, and is read once: its largest logit m, the sum s of exp(x - m), then the
// gradient.  The loss alone is formed as the row streams by, with a running maximum; so
// is that of longer rows, which are read again for their gradient.
// The loss is log s - (x_target - m), which loses nothing where the
// target is all but certain, as lse - x_target would.

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <string>

#include "../../include/mtdao_ops.h"
#include "host.hpp"
#include "ops_device.hpp"

using namespace mtdao;
using namespace mtdao::ops;

namespace {

template <typename T>
constexpr int kE = 16 / (int)sizeof(T);  // elements of a thread's vector: 16 bytes
constexpr int kFinish = 1024;  // threads of the kernels over all rows
constexpr int kOneEach = 256;  // rows of which each has a CU

struct Args {
  int64_t rows, cols, ld, ld_d;
  const void *logits, *targets;
  const float* d_loss;
  float* losses;
  void* d_logits;
  const float* weight;  // of a row's gradient: 1 / rows with a target (mean)
  float z, scale;
  int32_t wide;         // targets have 64 bits
  int32_t each;         // d_loss has a number for each row
};

// Largest and sum over the THREADS threads of a row (a wave, or the workgroup), in each.
template <int THREADS>
__device__ __forceinline__ float row_max(float x, float* part) {
  x = max_with32(max32(x));
  if constexpr (THREADS > 64) {
    __syncthreads();
    if (threadIdx.x % 64 == 0) part[threadIdx.x / 64] = x;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < THREADS / 64; ++w) x = fmaxf(x, part[w]);
  }
  return x;
}
template <int THREADS>
__device__ __forceinline__ float row_sum(float x, float* part) {
  x = sum64(x);
  if constexpr (THREADS > 64) {
    __syncthreads();
    if (threadIdx.x % 64 == 0) part[threadIdx.x / 64] = x;
    __syncthreads();
    x = 0.0f;
#pragma unroll
    for (int w = 0; w < THREADS / 64; ++w) x += part[w];
  }
  return x;
}

constexpr float kLog2e = 1.44269504f;
__device__ __forceinline__ float exp_of(float x) { return __builtin_amdgcn_exp2f(x * kLog2e); }

// A vector as it is in memory.  (Of fp32 four: with eight, two loads apart by a lane's 32
// bytes, 2047 x 32003 took 139 us.)
template <typename T, bool NT>
struct Vector : Raw<T, NT> {};
template <bool NT>
struct Vector<float, NT> {
  float w[4];
  __device__ __forceinline__ void load(const float* p, int n) { load_some<4, NT>(p, n, w); }
  __device__ __forceinline__ void values(float (&o)[4]) const {
#pragma unroll
    for (int t = 0; t < 4; ++t) o[t] = w[t];
  }
};

// A vector's logits, minus infinity from n on.
template <typename R, int N>
__device__ __forceinline__ void logits_of(const R& raw, int n, float (&v)[N]) {
  raw.values(v);
  if (n < N) {
#pragma unroll
    for (int t = 0; t < N; ++t)
      if (t >= n) v[t] = -INFINITY;
  }
}

// What a row's target asks for.
template <typename T>
struct Target {
  int64_t at;   // < 0: nothing
  bool known;
  float x;      // its logit
  __device__ __forceinline__ Target(const Args& a, const T* x, int64_t row) : at(id_of(a.targets, a.wide, row)) {
    known = at < a.cols;
    this->x = at < 0 ? 0.0f : known ? to_f32(x[at]) : NAN;
  }
};

// The row's loss from m and s (one thread stores it), and the factors of its gradient: of exp(x - m) and of the target.
struct Weights {
  float each, target;
};
template <typename T>
__device__ __forceinline__ Weights weights_of(const Args& a, const Target<T>& target, int64_t row, float m, float s, bool stores) {
  const float log_s = logf(s), lse = m + log_s;
  if (a.losses && stores) a.losses[row] = log_s - (target.x - m) + (a.z != 0.0f ? a.z * lse * lse : 0.0f);
  float w = a.scale;
  if (a.weight) w *= *a.weight;
  if (a.d_loss) w *= a.d_loss[a.each ? row : 0];
  if (!target.known) w = NAN;
  return {w * (a.z != 0.0f ? 1.0f + 2.0f * a.z * lse : 1.0f) / s, w};
}

// A vector of the gradient (the first n elements), the target's counted from the first.
template <bool NT, typename T, int N>
__device__ __forceinline__ void store_gradient(T* d, int n, float (&v)[N], float m, const Weights& w, int64_t target) {
#pragma unroll
  for (int t = 0; t < N; ++t) v[t] = w.each * exp_of(v[t] - m);
  if (target >= 0 && target < N) {
#pragma unroll
    for (int t = 0; t < N; ++t)
      if (t == target) v[t] -= w.target;
  }
  store_some<N, NT>(d, n, v);
}

// Nothing is asked of the row, and nothing of it is read.
template <int THREADS, typename T>
__device__ __forceinline__ void store_nothing(const Args& a, T* d, int64_t row, int tid) {
  if (a.losses && tid == 0) a.losses[row] = 0.0f;
  constexpr int N = kE<T>;
  const float none[N] = {};
  if (d)
    for (int64_t e = tid * N; e < a.cols; e += THREADS * N) store_some<N>(d + e, a.cols - e > N ? N : (int)(a.cols - e), none);
}

// Rows in registers: THREADS threads (64: four rows a workgroup) with NV vectors each.  Where
// they fit 64 registers two workgroups share a CU, and one's loads fill the other's sums and stores.
// Bound by HBM: 16384 x 50304 bf16 576 us, 5.7 TB/s; 2047 x 32003 fp32 94 us, 5.3 TB/s (three passes over
// memory took 996 and 196 us).  Loads and stores are non-temporal: 4096 x 50304 bf16 behind what wrote the
// logits 156 us in place of 167, smaller ones the same either way.
template <typename T, int THREADS, int NV>
__global__ __launch_bounds__(THREADS > 64 ? THREADS : 4 * THREADS, NV <= (sizeof(T) == 2 ? 7 : 8) ? 8 : 4) void k_cross_entropy_held(Args a) {
  __shared__ float part[THREADS / 64];
  constexpr int N = kE<T>, kRows = THREADS > 64 ? 1 : 4, kApart = THREADS * N;
  const int tid = (int)threadIdx.x % THREADS;
  const int64_t row = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * kRows + (int)threadIdx.x / THREADS;
  if (row >= a.rows) return;
  const T* x = reinterpret_cast<const T*>(a.logits) + row * a.ld;
  T* d = a.d_logits ? reinterpret_cast<T*>(a.d_logits) + row * a.ld_d : nullptr;
  const Target<T> target(a, x, row);
  if (target.at < 0) return store_nothing<THREADS>(a, d, row, tid);
  const int left = (int)a.cols - tid * N;  // elements from the thread's first vector on
  x += tid * N;
  Vector<T, true> raw[NV];
#pragma unroll
  for (int k = 0; k < NV; ++k) raw[k].load(x + k * kApart, left - k * kApart);
  float m = -INFINITY, v[N];
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    if (left > k * kApart) {
      logits_of(raw[k], left - k * kApart, v);
#pragma unroll
      for (int t = 0; t < N; ++t) m = fmaxf(m, v[t]);
    }
  }
  m = row_max<THREADS>(m, part);
  float s = 0.0f;
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    if (left > k * kApart) {
      logits_of(raw[k], left - k * kApart, v);
#pragma unroll
      for (int t = 0; t < N; ++t) s += exp_of(v[t] - m);
    }
  }
  s = row_sum<THREADS>(s, part);
  const Weights w = weights_of(a, target, row, m, s, tid == 0);
  if (!d) return;
  d += tid * N;
  const int at = target.known ? (int)target.at - tid * N : -1;
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    const int n = left - k * kApart;
    if (n > 0) {
      logits_of(raw[k], n, v);
      store_gradient<true>(d + k * kApart, n, v, m, w, at - k * kApart);
    }
  }
}

// Rows that stream by.  Each thread keeps the largest of its logits so far and the sum of exp(x - it).
// Bound by HBM: losses of 4096 x 50304 bf16 77 us, 5.3 TB/s.
template <typename T, int THREADS>
__global__ __launch_bounds__(THREADS) void k_cross_entropy(Args a) {
  __shared__ float part[THREADS / 64];
  constexpr int N = kE<T>, kAtOnce = 16 / N * 2;
  const int tid = (int)threadIdx.x;
  const int64_t row = (int64_t)blockIdx.y * gridDim.x + blockIdx.x;
  if (row >= a.rows) return;
  const T* x = reinterpret_cast<const T*>(a.logits) + row * a.ld;
  T* d = a.d_logits ? reinterpret_cast<T*>(a.d_logits) + row * a.ld_d : nullptr;
  const Target<T> target(a, x, row);
  if (target.at < 0) return store_nothing<THREADS>(a, d, row, tid);
  float mine = -INFINITY, s = 0.0f, v[N];
  for (int64_t from = 0; from < a.cols; from += kAtOnce * THREADS * N) {
    Vector<T, false> raw[kAtOnce];
    int n[kAtOnce];
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k) {
      const int64_t e = from + (k * THREADS + tid) * N, left = a.cols - e;
      n[k] = left > N ? N : left < 0 ? 0 : (int)left;
      raw[k].load(x + e, n[k]);
    }
    float most = mine;
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k) {
      logits_of(raw[k], n[k], v);
#pragma unroll
      for (int t = 0; t < N; ++t) most = fmaxf(most, v[t]);
    }
    if (most > mine) {
      s *= exp_of(mine - most);
      mine = most;
    }
    const float base = mine == -INFINITY ? 0.0f : mine;  // (nothing above minus infinity so far: terms of 0, not NaN)
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k) {
      logits_of(raw[k], n[k], v);
#pragma unroll
      for (int t = 0; t < N; ++t) s += exp_of(v[t] - base);
    }
  }
  const float m = row_max<THREADS>(mine, part);
  // (of a thread without a logit, or with none above minus infinity, s is 0; where no thread has one it is NaN)
  s = row_sum<THREADS>(mine > -INFINITY ? s * exp_of(mine - m) : m > -INFINITY ? s : NAN, part);
  const Weights w = weights_of(a, target, row, m, s, tid == 0);
  if (!d) return;
  for (int64_t e = tid * N; e < a.cols; e += THREADS * N) {
    const int n = a.cols - e > N ? N : (int)(a.cols - e);
    Vector<T, false> raw;
    raw.load(x + e, n);
    logits_of(raw, n, v);
    store_gradient<false>(d + e, n, v, m, w, target.at - e);
  }
}

// One over the number of rows with a target (1 where there is none).
__global__ __launch_bounds__(kFinish) void k_cross_entropy_count(const void* targets, int32_t wide, int64_t rows, float* weight) {
  __shared__ int64_t part[kFinish / 64];
  int64_t n = 0;
#pragma unroll 8
  for (int64_t i = threadIdx.x; i < rows; i += kFinish) n += id_of(targets, wide, i) >= 0;
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) n += __shfl_xor(n, o);
  if (threadIdx.x % 64 == 0) part[threadIdx.x / 64] = n;
  __syncthreads();
  if (threadIdx.x == 0) {
    n = 0;
    for (int w = 0; w < kFinish / 64; ++w) n += part[w];
    *weight = (float)(1.0 / (double)(n > 0 ? n : 1));
  }
}

// The sum of the rows' losses, or their mean over rows with a target.
__global__ __launch_bounds__(kFinish) void k_cross_entropy_sum(const float* losses, const void* targets, int32_t wide, int64_t rows, int32_t mean,
                                                               float* loss) {
  __shared__ double part[kFinish / 64];
  __shared__ int64_t counted[kFinish / 64];
  double sum = 0.0;
  int64_t n = 0;
#pragma unroll 8
  for (int64_t i = threadIdx.x; i < rows; i += kFinish) {
    sum += losses[i];
    n += id_of(targets, wide, i) >= 0;
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) {
    sum += __shfl_xor(sum, o);
    n += __shfl_xor(n, o);
  }
  if (threadIdx.x % 64 == 0) {
    part[threadIdx.x / 64] = sum;
    counted[threadIdx.x / 64] = n;
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    sum = 0.0;
    n = 0;
    for (int w = 0; w < kFinish / 64; ++w) {
      sum += part[w];
      n += counted[w];
    }
    *loss = (float)(mean && n > 0 ? sum / (double)n : sum);
  }
}

// --------------------------------------------------------------------- host

int32_t check(const mtdao_cross_entropy_args* a, std::string* e) {
  if (!a) return fail(e, MTDAO_ERR_INVALID_ARG, "args is NULL");
  if (a->rows < 0 || a->rows > (INT64_C(1) << 31)) return fail(e, MTDAO_ERR_INVALID_ARG, "rows %lld: 0..2^31", (long long)a->rows);
  if (a->cols < 1 || a->cols > (INT64_C(1) << 31)) return fail(e, MTDAO_ERR_INVALID_ARG, "cols %lld: 1..2^31", (long long)a->cols);
  if (a->dtype != MTDAO_F32 && a->dtype != MTDAO_BF16) return fail(e, MTDAO_ERR_INVALID_ARG, "dtype must be F32(0) or BF16(1)");
  if (a->target_bits != 32 && a->target_bits != 64) return fail(e, MTDAO_ERR_INVALID_ARG, "target_bits %d is not 32 or 64", a->target_bits);
  if (a->reduction != MTDAO_LOSS_NONE && a->reduction != MTDAO_LOSS_SUM && a->reduction != MTDAO_LOSS_MEAN)
    return fail(e, MTDAO_ERR_INVALID_ARG, "reduction %d is unknown", a->reduction);
  if (!std::isfinite(a->z_loss) || !std::isfinite(a->scale)) return fail(e, MTDAO_ERR_INVALID_ARG, "z_loss or scale is not finite");
  return MTDAO_OK;
}

int32_t check_pointers(const mtdao_cross_entropy_args& a, std::string* e) {
  if (a.loss && a.reduction == MTDAO_LOSS_NONE) return fail(e, MTDAO_ERR_INVALID_ARG, "loss needs a reduction");
  if (!a.losses && !a.loss && !a.d_logits) return fail(e, MTDAO_ERR_INVALID_ARG, "losses, loss and d_logits are all NULL");
  if (!aligned_to(a.losses, 4) || !aligned_to(a.loss, 4) || !aligned_to(a.d_loss, 4))
    return fail(e, MTDAO_ERR_ALIGN, "losses, loss or d_loss is not aligned to its element");
  if (a.rows == 0) return MTDAO_OK;
  const int64_t most = INT64_C(1) << 40, es = esize(a.dtype);
  if (a.ld_logits < a.cols || a.ld_logits > most / a.rows || (a.d_logits && (a.ld_d < a.cols || a.ld_d > most / a.rows)))
    return fail(e, MTDAO_ERR_INVALID_ARG, "a row stride is below the columns or exceeds 2^40 elements in all");
  if (!a.logits || !a.targets) return fail(e, MTDAO_ERR_INVALID_ARG, "logits or targets is NULL");
  if (!aligned_to(a.logits, (uintptr_t)es) || !aligned_to(a.d_logits, (uintptr_t)es) || !aligned_to(a.targets, (uintptr_t)a.target_bits / 8))
    return fail(e, MTDAO_ERR_ALIGN, "logits, d_logits or targets is not aligned to its element");
  if (a.d_logits) {
    const int64_t in = ((a.rows - 1) * a.ld_logits + a.cols) * es, out = ((a.rows - 1) * a.ld_d + a.cols) * es;
    if (overlap(a.logits, in, a.d_logits, out) && (a.logits != a.d_logits || a.ld_logits != a.ld_d))
      return fail(e, MTDAO_ERR_INVALID_ARG, "d_logits overlaps logits other than element on element");
  }
  // (the losses are written while other rows are read)
  struct { const void* p; int64_t bytes; bool written; } all[] = {
      {a.losses, a.rows * 4, true}, {a.loss, 4, true}, {a.d_logits, ((a.rows - 1) * a.ld_d + a.cols) * es, true},
      {a.logits, ((a.rows - 1) * a.ld_logits + a.cols) * es, false}, {a.targets, a.rows * a.target_bits / 8, false},
      {a.d_loss, a.reduction == MTDAO_LOSS_NONE ? a.rows * 4 : 4, false}};
  for (int i = 0; i < 6; ++i)
    for (int j = i + 1; j < 6; ++j)
      if (all[i].p && all[j].p && all[i].written && !(i == 2 && j == 3) && overlap(all[i].p, all[i].bytes, all[j].p, all[j].bytes))
        return fail(e, MTDAO_ERR_INVALID_ARG, "losses, loss or d_logits overlaps another operand");
  return MTDAO_OK;
}

template <typename T, int THREADS, int NV>
void launch_held(const Args& k, hipStream_t st) {
  constexpr int rows = THREADS > 64 ? 1 : 4;
  hipLaunchKernelGGL((k_cross_entropy_held<T, THREADS, NV>), grid_of((k.rows + rows - 1) / rows), dim3(THREADS * rows), 0, st, k);
}
template <typename T>
void launch_rows(const Args& k, hipStream_t st) {
  const int64_t c = k.cols;
  // Threads and vectors that hold the row: a wave while it does so with at most 32 logits a lane, then as few threads as do so with
  // 32 each.  Loss and gradient in us by two forms (threads x vectors of eight), first of 64 rows, then of 0.4 to 0.8 GB of rows:
  //   columns                     bf16               fp32
  //     512   64 x 1,  256 x 1    5.2 4.2,  42  94   4.3  4.0,  49  97
  //    2048   64 x 4,  256 x 1    5.4 4.1,  92 147   6.0  4.3, 180 171
  //    4096   64 x 8,  256 x 2    7.5 4.5, 179 198   8.3  4.8, 284 261
  //    8192  256 x 4,  512 x 2    5.5 4.8, 265 293   6.0  5.1, 265 276
  //   16384  256 x 8,  512 x 4    7.7 6.1, 282 279   8.6  6.7, 298 285
  //   32768  512 x 8, 1024 x 4    8.8 8.0, 300 311  10.7  9.9, 281 295
  //   57344 1024 x 7, 1024 x 8   11.7 12.0, 297 350  14.8 15.0, 314 317   (streaming, read twice: 13.1, 379; 16.1, 373)
  // Without a gradient rows of more than 8192 stream.  Streaming and held: 0.8 GB of 16384 columns bf16 147 147, fp32 162 151, of 50304
  // 166 142 and 164 176; 64 rows of 50304 8.5 7.7 and 8.7 10.2.
  constexpr int W = 8 / kE<T>;  // vectors of eight elements
  if (c <= 512) return launch_held<T, 64, W>(k, st);
  if (c <= 1024) return launch_held<T, 64, 2 * W>(k, st);
  if (c <= 2048) return launch_held<T, 64, 4 * W>(k, st);
  if (c <= 4096) return launch_held<T, 256, 2 * W>(k, st);
  if (c <= 8192) return launch_held<T, 256, 4 * W>(k, st);
  if (k.d_logits) {
    if (c <= 16384) return launch_held<T, 512, 4 * W>(k, st);
    if (c <= 32768) return launch_held<T, 1024, 4 * W>(k, st);
    if (c <= 57344) return launch_held<T, 1024, 7 * W>(k, st);
    if (c <= 65536) return launch_held<T, 1024, 8 * W>(k, st);
    if constexpr (sizeof(T) == 2) {
      if (c <= 131072) return launch_held<T, 1024, 16>(k, st);
    }
  }
  // Up to a row a CU more threads each, which takes fewer turns of the loop.  Losses in us, 256 / 1024 threads, bf16: 64 x 32003
  // 8.4 / 6.7, 256 x 50304 12.5 / 10.2, 257 x 50304 12.6 / 14.7, 384 x 32003 10.1 / 12.4, 1024 x 9000 10 / 21 (and 256 x 9000 6.8 / 7.2); fp32:
  // 256 x 32003 10.4 / 9.3, 257 x 32003 10.5 / 12.7.  With a gradient, which reads the row twice, always: 2000 x 140000 bf16 358 / 284,
  // 512 x 70000 fp32 108 / 87.
  if (k.rows <= kOneEach || k.d_logits) hipLaunchKernelGGL((k_cross_entropy<T, 1024>), grid_of(k.rows), dim3(1024), 0, st, k);
  else hipLaunchKernelGGL((k_cross_entropy<T, 256>), grid_of(k.rows), dim3(256), 0, st, k);
}

struct Layout {
  size_t losses, weight, bytes;
};
Layout layout_of(const mtdao_cross_entropy_args& a) {
  if (a.reduction == MTDAO_LOSS_NONE) return {0, 0, 0};
  return {0, up256((size_t)a.rows * sizeof(float)), up256((size_t)a.rows * sizeof(float)) + 256};
}

}  // namespace

extern "C" {

int32_t mtdao_cross_entropy_workspace_bytes(const mtdao_cross_entropy_args* a, size_t* bytes) {
  const int32_t r = check(a, &g_err);
  if (r != MTDAO_OK) return r;
  if (!bytes) return fail(&g_err, MTDAO_ERR_INVALID_ARG, "bytes is NULL");
  *bytes = layout_of(*a).bytes;
  return MTDAO_OK;
}

int32_t mtdao_cross_entropy(const mtdao_cross_entropy_args* args, void* workspace, size_t workspace_bytes, void* hip_stream) {
  std::string* e = &g_err;
  int32_t r = check(args, e);
  if (r == MTDAO_OK) r = check_pointers(*args, e);
  if (r != MTDAO_OK) return r;
  const mtdao_cross_entropy_args& a = *args;
  const Layout l = layout_of(a);
  if (l.bytes > 0 && (!workspace || workspace_bytes < l.bytes))
    return fail(e, MTDAO_ERR_WORKSPACE, "workspace of %zu bytes required, %zu given", l.bytes, workspace ? workspace_bytes : (size_t)0);
  if (l.bytes > 0 && !aligned_to(workspace, 256)) return fail(e, MTDAO_ERR_ALIGN, "workspace is not 256-byte aligned");
  char* w = static_cast<char*>(workspace);
  hipStream_t st = reinterpret_cast<hipStream_t>(hip_stream);
  RoctxRange range("mtdao_cross_entropy %lld x %lld", (long long)a.rows, (long long)a.cols);
  Args k = {a.rows, a.cols, a.ld_logits, a.ld_d, a.logits, a.targets, a.d_loss, a.losses, a.d_logits, nullptr, a.z_loss, a.scale, a.target_bits == 64,
            a.reduction == MTDAO_LOSS_NONE};
  if (a.loss && !k.losses) k.losses = reinterpret_cast<float*>(w + l.losses);
  if (a.rows > 0) {
    if (a.d_logits && a.reduction == MTDAO_LOSS_MEAN) {
      float* weight = reinterpret_cast<float*>(w + l.weight);
      hipLaunchKernelGGL(k_cross_entropy_count, dim3(1), dim3(kFinish), 0, st, a.targets, k.wide, a.rows, weight);
      k.weight = weight;
    }
    if (a.dtype == MTDAO_BF16) launch_rows<bf16_t>(k, st);
    else launch_rows<float>(k, st);
  }
  if (a.loss)
    hipLaunchKernelGGL(k_cross_entropy_sum, dim3(1), dim3(kFinish), 0, st, k.losses, a.targets, k.wide, a.rows, (int32_t)(a.reduction == MTDAO_LOSS_MEAN),
                       a.loss);
  return hip_check(e, hipGetLastError(), "mtdao_cross_entropy launch");
}

}  // extern "C"
