// Cross entropy of rows of logits and its gradient (include/mtdao_ops.h).
//
// A workgroup takes a row: its largest logit m, the sum s of exp(x - m), then the
// gradient.  The loss is log s - (x_target - m), which loses nothing where the
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

constexpr int kThreads = 256;
constexpr int kE = 8;          // elements of a thread's vector
constexpr int kFinish = 1024;  // threads of the kernels over all rows

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

__device__ __forceinline__ int64_t id_of(const void* ids, int32_t wide, int64_t i) {
  return wide ? reinterpret_cast<const int64_t*>(ids)[i] : (int64_t) reinterpret_cast<const int32_t*>(ids)[i];
}

// Largest and sum over the workgroup, in every thread.
template <int WAVES>
__device__ __forceinline__ float group_max(float x, float* part) {
  x = max_with32(max32(x));
  __syncthreads();
  if (threadIdx.x % 64 == 0) part[threadIdx.x / 64] = x;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < WAVES; ++w) x = fmaxf(x, part[w]);
  return x;
}
template <int WAVES>
__device__ __forceinline__ float group_sum(float x, float* part) {
  x = sum64(x);
  __syncthreads();
  if (threadIdx.x % 64 == 0) part[threadIdx.x / 64] = x;
  __syncthreads();
  x = 0.0f;
#pragma unroll
  for (int w = 0; w < WAVES; ++w) x += part[w];
  return x;
}

constexpr float kLog2e = 1.44269504f;
__device__ __forceinline__ float exp_of(float x) { return __builtin_amdgcn_exp2f(x * kLog2e); }

template <typename T>
__global__ __launch_bounds__(kThreads) void k_cross_entropy(Args a) {
  __shared__ float part[kThreads / 64];
  const int64_t row = (int64_t)blockIdx.y * gridDim.x + blockIdx.x;
  if (row >= a.rows) return;
  const T* x = reinterpret_cast<const T*>(a.logits) + row * a.ld;
  T* d = a.d_logits ? reinterpret_cast<T*>(a.d_logits) + row * a.ld_d : nullptr;
  const int64_t target = id_of(a.targets, a.wide, row);
  const float none[kE] = {};
  if (target < 0) {  // nothing is asked of this row, and nothing of it is read
    if (a.losses && threadIdx.x == 0) a.losses[row] = 0.0f;
    if (d)
      for (int64_t e = threadIdx.x * kE; e < a.cols; e += kThreads * kE) store_some<kE>(d + e, a.cols - e > kE ? kE : (int)(a.cols - e), none);
    return;
  }
  const bool known = target < a.cols;
  const float at_target = known ? to_f32(x[target]) : NAN;
  float m = -INFINITY, v[kE];
  for (int64_t e = threadIdx.x * kE; e < a.cols; e += kThreads * kE) {
    const int n = a.cols - e > kE ? kE : (int)(a.cols - e);
    load_some<kE>(x + e, n, v);
#pragma unroll
    for (int t = 0; t < kE; ++t)
      if (t < n) m = fmaxf(m, v[t]);
  }
  m = group_max<kThreads / 64>(m, part);
  float s = 0.0f;
  for (int64_t e = threadIdx.x * kE; e < a.cols; e += kThreads * kE) {
    const int n = a.cols - e > kE ? kE : (int)(a.cols - e);
    load_some<kE>(x + e, n, v);
#pragma unroll
    for (int t = 0; t < kE; ++t)
      if (t < n) s += exp_of(v[t] - m);
  }
  s = group_sum<kThreads / 64>(s, part);
  const float log_s = logf(s), lse = m + log_s;
  if (a.losses && threadIdx.x == 0) a.losses[row] = log_s - (at_target - m) + (a.z != 0.0f ? a.z * lse * lse : 0.0f);
  if (!d) return;
  float weight = a.scale;
  if (a.weight) weight *= *a.weight;
  if (a.d_loss) weight *= a.d_loss[a.each ? row : 0];
  if (!known) weight = NAN;
  const float of_each = weight * (1.0f + 2.0f * a.z * lse) / s;
  for (int64_t e = threadIdx.x * kE; e < a.cols; e += kThreads * kE) {
    const int n = a.cols - e > kE ? kE : (int)(a.cols - e);
    load_some<kE>(x + e, n, v);
#pragma unroll
    for (int t = 0; t < kE; ++t) v[t] = of_each * exp_of(v[t] - m) - (e + t == target ? weight : 0.0f);
    store_some<kE>(d + e, n, v);
  }
}

// One over the number of rows with a target (1 where there is none).
__global__ __launch_bounds__(kFinish) void k_cross_entropy_count(const void* targets, int32_t wide, int64_t rows, float* weight) {
  __shared__ int64_t part[kFinish / 64];
  int64_t n = 0;
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

size_t up256(size_t n) { return (n + 255) / 256 * 256; }
int64_t esize(int32_t dt) { return dt == MTDAO_BF16 ? 2 : 4; }

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
    if (overlap(a.targets, a.rows * a.target_bits / 8, a.d_logits, out)) return fail(e, MTDAO_ERR_INVALID_ARG, "d_logits overlaps targets");
  }
  return MTDAO_OK;
}

struct Layout {
  size_t losses, weight, bytes;
};
Layout layout_of(const mtdao_cross_entropy_args& a) {
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
  if (!workspace || workspace_bytes < l.bytes)
    return fail(e, MTDAO_ERR_WORKSPACE, "workspace of %zu bytes required, %zu given", l.bytes, workspace ? workspace_bytes : (size_t)0);
  if (!aligned_to(workspace, 256)) return fail(e, MTDAO_ERR_ALIGN, "workspace is not 256-byte aligned");
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
    if (a.dtype == MTDAO_BF16) hipLaunchKernelGGL(k_cross_entropy<bf16_t>, grid_of(a.rows), dim3(kThreads), 0, st, k);
    else hipLaunchKernelGGL(k_cross_entropy<float>, grid_of(a.rows), dim3(kThreads), 0, st, k);
  }
  if (a.loss)
    hipLaunchKernelGGL(k_cross_entropy_sum, dim3(1), dim3(kFinish), 0, st, k.losses, a.targets, k.wide, a.rows, (int32_t)(a.reduction == MTDAO_LOSS_MEAN),
                       a.loss);
  return hip_check(e, hipGetLastError(), "mtdao_cross_entropy launch");
}

}  // extern "C"
