// Matrices in 8-bit floating point with a scale per block of 128, and their
// product (include/mtdao_ops.h).

#include <hip/hip_runtime.h>

#include <algorithm>
#include <string>
#include <type_traits>

#include "../../include/mtdao_ops.h"
#include "host.hpp"
#include "ops_device.hpp"

using namespace mtdao;
using namespace mtdao::ops;

namespace {

// A matrix of 8-bit blocks as the kernels see it.
struct Mat {
  uint8_t* codes;
  uint8_t* scales;
  int64_t rows, ld;
  int32_t blocks, scale_ld;  // blocks of a row, and bytes from row to row of the scales
};

// --------------------------------------------------------------- quantizers

constexpr int kThreads = 256;
constexpr int kE = 8;  // elements of a thread's vector: 16 threads hold a block

// Blocks along the rows: sixteen of a workgroup, in the order of the scales.
template <typename T>
__global__ __launch_bounds__(kThreads) void k_quantize8_rows(const T* x, int64_t ld, int64_t cols, Mat q) {
  const int64_t b = (int64_t)blockIdx.x * (kThreads / 16) + threadIdx.x / 16;
  const int64_t row = b / q.scale_ld;
  const int kb = (int)(b - row * q.scale_ld), e = kb * kBlock8 + (int)(threadIdx.x % 16) * kE;
  float a[kE], most = 0.0f;
  const bool live = row < q.rows && kb < q.blocks;
  const int64_t n = live ? cols - e : 0;
  if (n > 0) {
    load_some<kE>(x + row * ld + e, n > kE ? kE : (int)n, a);
  } else {
#pragma unroll
    for (int t = 0; t < kE; ++t) a[t] = 0.0f;
  }
#pragma unroll
  for (int t = 0; t < kE; ++t) most = fmaxf(most, finite_abs(a[t]));
  const uint32_t byte = live ? scale_byte(max16(most)) : 127u;
  const float inv = inverse_scale_of(byte);
#pragma unroll
  for (int t = 0; t < kE; ++t) a[t] = nan_if_infinite(a[t] * inv);
  if (live) {
    uint2 c = {codes_of(a[0], a[1], a[2], a[3]), codes_of(a[4], a[5], a[6], a[7])};
    *reinterpret_cast<uint2*>(q.codes + row * q.ld + e) = c;
  }
  if (row < q.rows && threadIdx.x % 16 == 0) q.scales[row * q.scale_ld + kb] = (uint8_t)byte;
}

// A tile of 128 x 128: a thread holds eight rows of eight columns, so that a
// transposed row of codes is eight consecutive bytes of it.  SQUARE: one
// scale for the tile; else blocks along the rows for q, along the columns
// for qt, which goes through LDS to be written in whole lines.
template <typename T, bool SQUARE>
__global__ __launch_bounds__(kThreads) void k_quantize8_tile(const T* x, int64_t ld, int64_t cols, int64_t rows, Mat q,
                                                             Mat qt) {
  constexpr int kPad = kBlock8 + 16;
  __shared__ __attribute__((aligned(16))) uint8_t turned[kBlock8 * kPad];
  __shared__ float most[16][kBlock8];
  const int c8 = (int)(threadIdx.x % 16) * kE, r8 = (int)(threadIdx.x / 16) * 8;
  const int64_t row0 = (int64_t)blockIdx.y * kBlock8, col0 = (int64_t)blockIdx.x * kBlock8;
  const int64_t in_cols = cols - col0 - c8, in_rows = rows - row0 - r8;
  const int nc = in_cols < 0 ? 0 : in_cols > kE ? kE : (int)in_cols;
  float a[8][kE];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    if (i < in_rows && nc > 0) {
      load_some<kE>(x + (row0 + r8 + i) * ld + col0 + c8, nc, a[i]);
    } else {
#pragma unroll
      for (int t = 0; t < kE; ++t) a[i][t] = 0.0f;
    }
  }
  uint32_t row_byte[8];
  float all = 0.0f;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    float m = 0.0f;
#pragma unroll
    for (int t = 0; t < kE; ++t) m = fmaxf(m, finite_abs(a[i][t]));
    if constexpr (SQUARE) all = fmaxf(all, m);
    else row_byte[i] = scale_byte(max16(m));
  }
  uint32_t col_byte[kE];
  if constexpr (SQUARE) {
    all = max32(all);
    all = fmaxf(all, __shfl_xor(all, 32));
    if (threadIdx.x % 64 == 0) most[0][threadIdx.x / 64] = all;
    __syncthreads();
    const uint32_t byte = scale_byte(fmaxf(fmaxf(most[0][0], most[0][1]), fmaxf(most[0][2], most[0][3])));
#pragma unroll
    for (int i = 0; i < 8; ++i) row_byte[i] = col_byte[i] = byte;
  } else {
#pragma unroll
    for (int t = 0; t < kE; ++t) {
      float m = 0.0f;
#pragma unroll
      for (int i = 0; i < 8; ++i) m = fmaxf(m, finite_abs(a[i][t]));
      most[threadIdx.x / 16][c8 + t] = m;
    }
    __syncthreads();
#pragma unroll
    for (int t = 0; t < kE; ++t) {
      float m = 0.0f;
#pragma unroll
      for (int g = 0; g < 16; ++g) m = fmaxf(m, most[g][c8 + t]);
      col_byte[t] = scale_byte(m);
    }
  }
  if (q.codes) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float inv = inverse_scale_of(row_byte[i]);
      float s[kE];
#pragma unroll
      for (int t = 0; t < kE; ++t) s[t] = nan_if_infinite(a[i][t] * inv);
      if (i < in_rows) {
        uint2 c = {codes_of(s[0], s[1], s[2], s[3]), codes_of(s[4], s[5], s[6], s[7])};
        *reinterpret_cast<uint2*>(q.codes + (row0 + r8 + i) * q.ld + col0 + c8) = c;
      }
    }
    const bool last = blockIdx.x + 1 == gridDim.x;
    const int bytes = last ? q.scale_ld - (int)blockIdx.x : 1;  // the row's unused bytes too
    if constexpr (SQUARE) {
      if (threadIdx.x < (unsigned)bytes)
        q.scales[(int64_t)blockIdx.y * q.scale_ld + blockIdx.x + threadIdx.x] = threadIdx.x == 0 ? (uint8_t)row_byte[0] : 127;
    } else if (threadIdx.x % 16 == 0) {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (i < in_rows) {
          uint8_t* s = q.scales + (row0 + r8 + i) * q.scale_ld + blockIdx.x;
          for (int k = 0; k < bytes; ++k) s[k] = k == 0 ? (uint8_t)row_byte[i] : 127;
        }
    }
  }
  if (qt.codes) {
#pragma unroll
    for (int t = 0; t < kE; ++t) {
      const float inv = inverse_scale_of(col_byte[t]);
      float s[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) s[i] = nan_if_infinite(a[i][t] * inv);
      uint2 c = {codes_of(s[0], s[1], s[2], s[3]), codes_of(s[4], s[5], s[6], s[7])};
      *reinterpret_cast<uint2*>(turned + (c8 + t) * kPad + r8) = c;
    }
    const bool last = blockIdx.y + 1 == gridDim.y;
    const int bytes = last ? qt.scale_ld - (int)blockIdx.y : 1;
    if constexpr (SQUARE) {
      if (threadIdx.x < (unsigned)bytes)
        qt.scales[(int64_t)blockIdx.x * qt.scale_ld + blockIdx.y + threadIdx.x] = threadIdx.x == 0 ? (uint8_t)col_byte[0] : 127;
    } else if (threadIdx.x < 16) {
#pragma unroll
      for (int t = 0; t < kE; ++t)
        if (t < nc) {
          uint8_t* s = qt.scales + (col0 + c8 + t) * qt.scale_ld + blockIdx.y;
          for (int k = 0; k < bytes; ++k) s[k] = k == 0 ? (uint8_t)col_byte[t] : 127;
        }
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int at = k * kThreads + (int)threadIdx.x, r = at / 8, c = at % 8 * 16;
      if (col0 + r < cols)
        *reinterpret_cast<uint4*>(qt.codes + (col0 + r) * qt.ld + row0 + c) =
            *reinterpret_cast<const uint4*>(turned + r * kPad + c);
    }
  }
}

// ------------------------------------------------------------------ product
//
// Every matrix instruction takes 16 x 128 codes of each side and their
// scales: a block of 128 is its whole contraction, and as the scales are
// powers of two in the instruction's own format, sums stay in its
// accumulators from the first block to the last.  Which 16-byte chunks of a
// block a lane holds is free as long as both sides agree, since they share
// one scale.  Rows of b go in as the instruction's rows, so that a lane ends
// with four consecutive columns of a row of c.
//
// Within a group of products the 8-bit instructions drop what lies more than
// 13 bits below the largest one (measured: 65536 + 4 gives 65536, in the
// instruction with scales and the one without), which leaves sums 1.3e-5
// (normal values) to 4e-5 (outlier columns) off in relative norm.  For a bf16
// c that is a hundredth of its rounding.  An fp32 c is formed by bf16
// instructions instead, at half their rate: codes times scales are bf16
// values, and their products are summed in fp32.

typedef int v8i __attribute__((ext_vector_type(8)));
typedef int v4i __attribute__((ext_vector_type(4)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef __bf16 v2bf __attribute__((ext_vector_type(2)));
typedef __bf16 v8bf __attribute__((ext_vector_type(8)));

struct Product {
  Mat a, b;
  void* c;
  int64_t ldc;
  int32_t a_scale_rows, b_scale_rows, accumulate;
};

// A 128-byte row of a tile in LDS: its eight 16-byte chunks, at the places
// that eight consecutive rows need to be read from different banks.
__device__ __forceinline__ int chunk_at(int row, int chunk) { return row * 128 + ((chunk ^ (row & 7)) << 4); }

__device__ __forceinline__ v8i fragment(const uint8_t* tile, int row, int group) {
  const v4i lo = *reinterpret_cast<const v4i*>(tile + chunk_at(row, group));
  const v4i hi = *reinterpret_cast<const v4i*>(tile + chunk_at(row, group + 4));
  return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
}

// Eight codes (two of a fragment's words) times their scale, as bf16: exact
// down to bf16's smallest values.
__device__ __forceinline__ v8bf widened(v8i f, int part, float scale) {
  v8bf o;
#pragma unroll
  for (int w = 0; w < 2; ++w) {
    const v2bf lo = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((unsigned)f[2 * part + w], scale, false);
    const v2bf hi = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((unsigned)f[2 * part + w], scale, true);
    o[4 * w] = lo[0];
    o[4 * w + 1] = lo[1];
    o[4 * w + 2] = hi[0];
    o[4 * w + 3] = hi[1];
  }
  return o;
}

__device__ __forceinline__ __amdgpu_buffer_rsrc_t buffer_of(const uint8_t* p, int64_t bytes) {
  const int64_t most = INT64_C(0x7fffffff);
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(p), 0, (int)(bytes < most ? bytes : most), 0x00027000);
}

template <int BM, int BN, typename CT>
__global__ __launch_bounds__(256) void k_product8(Product p) {
  constexpr int kWM = BM / 2, kWN = BN / 2, kMI = kWM / 16, kNI = kWN / 16;
  __shared__ __attribute__((aligned(1024))) uint8_t ta[BM * 128];
  __shared__ __attribute__((aligned(1024))) uint8_t tb[BN * 128];
  const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const int64_t row0 = (int64_t)blockIdx.y * BM, col0 = (int64_t)blockIdx.x * BN;
  const auto ra = buffer_of(p.a.codes + row0 * p.a.ld, (p.a.rows - row0) * p.a.ld);
  const auto rb = buffer_of(p.b.codes + col0 * p.b.ld, (p.b.rows - col0) * p.b.ld);
  // a wave loads eight rows at once: lane l the chunk that belongs at place l % 8 of row l / 8
  const int lr = lane / 8, lc = (lane % 8) ^ (lr & 7);
  const int wm = wave / 2 * kWM, wn = wave % 2 * kWN, fr = lane % 16, fg = lane / 16;
  const uint8_t *sa[kMI], *sb[kNI];
#pragma unroll
  for (int i = 0; i < kMI; ++i) {
    const int64_t r = row0 + wm + i * 16 + fr;
    sa[i] = p.a.scales + (r < p.a.rows ? r : p.a.rows - 1) / p.a_scale_rows * p.a.scale_ld;
  }
#pragma unroll
  for (int j = 0; j < kNI; ++j) {
    const int64_t r = col0 + wn + j * 16 + fr;
    sb[j] = p.b.scales + (r < p.b.rows ? r : p.b.rows - 1) / p.b_scale_rows * p.b.scale_ld;
  }
  v4f acc[kMI][kNI];
#pragma unroll
  for (int i = 0; i < kMI; ++i)
#pragma unroll
    for (int j = 0; j < kNI; ++j) acc[i][j] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
  for (int kb = 0; kb < p.a.blocks; ++kb) {
    for (int r = wave * 8; r < BM; r += 32)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(ra, (__attribute__((address_space(3))) void*)(ta + r * 128), 16,
                                               (r + lr) * (int)p.a.ld + lc * 16, kb * 128, 0, 0);
    for (int r = wave * 8; r < BN; r += 32)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rb, (__attribute__((address_space(3))) void*)(tb + r * 128), 16,
                                               (r + lr) * (int)p.b.ld + lc * 16, kb * 128, 0, 0);
    __syncthreads();
    v8i fb[kNI];
    int eb[kNI];
#pragma unroll
    for (int j = 0; j < kNI; ++j) {
      fb[j] = fragment(tb, wn + j * 16 + fr, fg);
      eb[j] = sb[j][kb];
    }
#pragma unroll
    for (int i = 0; i < kMI; ++i) {
      const v8i fa = fragment(ta, wm + i * 16 + fr, fg);
      const int ea = sa[i][kb];
      if constexpr (sizeof(CT) == 2) {
#pragma unroll
        for (int j = 0; j < kNI; ++j)
          acc[i][j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(fb[j], fa, acc[i][j], 0, 0, 0, eb[j], 0, ea);
      } else {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const v8bf wa = widened(fa, k, scale_of((uint32_t)ea));
#pragma unroll
          for (int j = 0; j < kNI; ++j)
            acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widened(fb[j], k, scale_of((uint32_t)eb[j])), wa, acc[i][j], 0, 0, 0);
        }
      }
    }
    __syncthreads();
  }
  CT* c = reinterpret_cast<CT*>(p.c);
#pragma unroll
  for (int i = 0; i < kMI; ++i) {
    const int64_t row = row0 + wm + i * 16 + fr;
    if (row >= p.a.rows) continue;
#pragma unroll
    for (int j = 0; j < kNI; ++j) {
      const int64_t col = col0 + wn + j * 16 + fg * 4, left = p.b.rows - col;
      if (left <= 0) continue;
      const int n = left > 4 ? 4 : (int)left;
      CT* to = c + row * p.ldc + col;
      float o[4] = {acc[i][j][0], acc[i][j][1], acc[i][j][2], acc[i][j][3]};
      if (p.accumulate) {
        float before[4];
        load_some<4>(to, n, before);
#pragma unroll
        for (int t = 0; t < 4; ++t) o[t] += before[t];
      }
      store_some<4>(to, n, o);
    }
  }
}

// --------------------------------------------------------------------- host

int64_t up(int64_t n, int64_t m) { return (n + m - 1) / m * m; }

constexpr int64_t kMostCols = INT64_C(1) << 22;  // a tile's rows stay within 2^31 bytes

int32_t check_matrix(const mtdao_matrix8& q, const char* name, std::string* e) {
  if (q.rows < 0 || q.cols < 0) return fail(e, MTDAO_ERR_INVALID_ARG, "%s: rows or cols < 0", name);
  if (q.cols > kMostCols) return fail(e, MTDAO_ERR_INVALID_ARG, "%s: cols exceed 2^22", name);
  if (q.rows > INT64_C(0x7fffffff)) return fail(e, MTDAO_ERR_INVALID_ARG, "%s: rows exceed 2^31", name);
  if (q.ld != up(q.cols, kBlock8)) return fail(e, MTDAO_ERR_INVALID_ARG, "%s: ld is not cols rounded up to 128", name);
  if (q.scale_ld != up(q.ld / kBlock8, 4))
    return fail(e, MTDAO_ERR_INVALID_ARG, "%s: scale_ld is not ld / 128 rounded up to 4", name);
  if (q.scale_rows != 1 && q.scale_rows != kBlock8)
    return fail(e, MTDAO_ERR_INVALID_ARG, "%s: scale_rows is not 1 or 128", name);
  if (q.rows > 0 && q.cols > 0) {
    if (!q.codes || !q.scales) return fail(e, MTDAO_ERR_INVALID_ARG, "%s: codes or scales is NULL", name);
    if (!aligned16(q.codes)) return fail(e, MTDAO_ERR_ALIGN, "%s: codes are not 16-byte aligned", name);
    if (!aligned_to(q.scales, 4)) return fail(e, MTDAO_ERR_ALIGN, "%s: scales are not 4-byte aligned", name);
  }
  return MTDAO_OK;
}

Mat mat_of(const mtdao_matrix8* q) {
  Mat m = {};
  if (!q) return m;
  m.codes = q->codes;
  m.scales = q->scales;
  m.rows = q->rows;
  m.ld = q->ld;
  m.blocks = (int32_t)(q->ld / kBlock8);
  m.scale_ld = (int32_t)q->scale_ld;
  return m;
}

int64_t scale_bytes(const mtdao_matrix8& q) { return (q.rows + q.scale_rows - 1) / q.scale_rows * q.scale_ld; }

}  // namespace

extern "C" {

int32_t mtdao_quantize8(const void* x, int32_t dtype, int64_t ld, const mtdao_matrix8* q, const mtdao_matrix8* qt,
                        void* hip_stream) {
  std::string* e = &g_err;
  if (!q && !qt) return fail(e, MTDAO_ERR_INVALID_ARG, "q and qt are NULL");
  if (dtype != MTDAO_F32 && dtype != MTDAO_BF16) return fail(e, MTDAO_ERR_INVALID_ARG, "dtype must be F32(0) or BF16(1)");
  int32_t r = MTDAO_OK;
  if (q) r = check_matrix(*q, "q", e);
  if (r == MTDAO_OK && qt) r = check_matrix(*qt, "qt", e);
  if (r != MTDAO_OK) return r;
  if (q && qt && (q->rows != qt->cols || q->cols != qt->rows || q->scale_rows != qt->scale_rows))
    return fail(e, MTDAO_ERR_INVALID_ARG, "qt is not q transposed");
  const int64_t rows = q ? q->rows : qt->cols, cols = q ? q->cols : qt->rows;
  if (rows == 0 || cols == 0) return MTDAO_OK;
  const int64_t es = dtype == MTDAO_BF16 ? 2 : 4;
  if (ld < cols || ld > (INT64_C(1) << 40) / rows)
    return fail(e, MTDAO_ERR_INVALID_ARG, "row stride %lld of x is below cols or exceeds 2^40 elements in all", (long long)ld);
  if (!x) return fail(e, MTDAO_ERR_INVALID_ARG, "x is NULL");
  if (!aligned_to(x, (uintptr_t)es)) return fail(e, MTDAO_ERR_ALIGN, "x is not aligned to its element");
  const int64_t xbytes = ((rows - 1) * ld + cols) * es;
  const mtdao_matrix8* outs[2] = {q, qt};
  for (const mtdao_matrix8* o : outs)
    if (o && (overlap(x, xbytes, o->codes, o->rows * o->ld) || overlap(x, xbytes, o->scales, scale_bytes(*o))))
      return fail(e, MTDAO_ERR_INVALID_ARG, "x overlaps an output");
  hipStream_t st = reinterpret_cast<hipStream_t>(hip_stream);
  RoctxRange range("mtdao_quantize8 rows=%lld cols=%lld", (long long)rows, (long long)cols);
  const Mat m = mat_of(q), mt = mat_of(qt);
  const bool square = (q ? q : qt)->scale_rows == kBlock8;
  auto with = [&](auto t) {
    using T = decltype(t);
    const T* in = static_cast<const T*>(x);
    if (!qt && !square) {
      const int64_t wgs = (rows * m.scale_ld + kThreads / 16 - 1) / (kThreads / 16);
      if (wgs > INT64_C(0x7fffff)) return false;
      hipLaunchKernelGGL(k_quantize8_rows<T>, dim3((unsigned)wgs), dim3(kThreads), 0, st, in, ld, cols, m);
      return true;
    }
    const int64_t ty = up(rows, kBlock8) / kBlock8;
    if (ty > 65535) return false;
    const dim3 grid((unsigned)(up(cols, kBlock8) / kBlock8), (unsigned)ty);
    if (square) hipLaunchKernelGGL((k_quantize8_tile<T, true>), grid, dim3(kThreads), 0, st, in, ld, cols, rows, m, mt);
    else hipLaunchKernelGGL((k_quantize8_tile<T, false>), grid, dim3(kThreads), 0, st, in, ld, cols, rows, m, mt);
    return true;
  };
  if (!(dtype == MTDAO_BF16 ? with(bf16_t{}) : with(float{})))
    return fail(e, MTDAO_ERR_INVALID_ARG, "the matrix exceeds the largest launch");
  return hip_check(e, hipGetLastError(), "mtdao_quantize8 launch");
}

int32_t mtdao_product8_workspace_bytes(int64_t m, int64_t n, int64_t k, size_t* bytes) {
  if (!bytes) return fail(&g_err, MTDAO_ERR_INVALID_ARG, "bytes is NULL");
  if (m < 0 || n < 0 || k < 0) return fail(&g_err, MTDAO_ERR_INVALID_ARG, "a size is below 0");
  *bytes = 0;
  return MTDAO_OK;
}

int32_t mtdao_product8(const mtdao_matrix8* a, const mtdao_matrix8* b, void* c, int32_t c_dtype, int64_t ldc,
                       int32_t accumulate, void* workspace, size_t workspace_bytes, void* hip_stream) {
  std::string* e = &g_err;
  if (!a || !b) return fail(e, MTDAO_ERR_INVALID_ARG, "a or b is NULL");
  int32_t r = check_matrix(*a, "a", e);
  if (r == MTDAO_OK) r = check_matrix(*b, "b", e);
  if (r != MTDAO_OK) return r;
  if (a->cols != b->cols) return fail(e, MTDAO_ERR_INVALID_ARG, "a has %lld columns, b has %lld", (long long)a->cols, (long long)b->cols);
  if (c_dtype != MTDAO_F32 && c_dtype != MTDAO_BF16) return fail(e, MTDAO_ERR_INVALID_ARG, "c_dtype must be F32(0) or BF16(1)");
  if (accumulate && c_dtype != MTDAO_F32) return fail(e, MTDAO_ERR_INVALID_ARG, "accumulate needs an fp32 c");
  if (a->rows == 0 || b->rows == 0) return MTDAO_OK;
  const int64_t es = c_dtype == MTDAO_BF16 ? 2 : 4;
  if (ldc < b->rows || ldc > (INT64_C(1) << 40) / a->rows)
    return fail(e, MTDAO_ERR_INVALID_ARG, "ldc %lld is below the columns of c or exceeds 2^40 elements in all", (long long)ldc);
  if (!c) return fail(e, MTDAO_ERR_INVALID_ARG, "c is NULL");
  if (!aligned_to(c, (uintptr_t)es)) return fail(e, MTDAO_ERR_ALIGN, "c is not aligned to its element");
  const int64_t cbytes = ((a->rows - 1) * ldc + b->rows) * es;
  for (const mtdao_matrix8* m : {a, b})
    if (overlap(c, cbytes, m->codes, m->rows * m->ld) || overlap(c, cbytes, m->scales, scale_bytes(*m)))
      return fail(e, MTDAO_ERR_INVALID_ARG, "c overlaps a or b");
  size_t need = 0;
  mtdao_product8_workspace_bytes(a->rows, b->rows, a->cols, &need);
  if (need > 0 && (!workspace || workspace_bytes < need))
    return fail(e, MTDAO_ERR_WORKSPACE, "workspace of %zu bytes required, %zu given", need, workspace ? workspace_bytes : (size_t)0);
  Product p = {};
  p.a = mat_of(a);
  p.b = mat_of(b);
  p.c = c;
  p.ldc = ldc;
  p.a_scale_rows = a->scale_rows;
  p.b_scale_rows = b->scale_rows;
  p.accumulate = accumulate;
  hipStream_t st = reinterpret_cast<hipStream_t>(hip_stream);
  RoctxRange range("mtdao_product8 m=%lld n=%lld k=%lld", (long long)a->rows, (long long)b->rows, (long long)a->cols);
  constexpr int B = 128;
  const int64_t ty = up(a->rows, B) / B;
  if (ty > 65535) return fail(e, MTDAO_ERR_INVALID_ARG, "the rows of a exceed the largest launch");
  const dim3 grid((unsigned)(up(b->rows, B) / B), (unsigned)ty);
  if (c_dtype == MTDAO_F32) hipLaunchKernelGGL((k_product8<B, B, float>), grid, dim3(256), 0, st, p);
  else hipLaunchKernelGGL((k_product8<B, B, bf16_t>), grid, dim3(256), 0, st, p);
  return hip_check(e, hipGetLastError(), "mtdao_product8 launch");
}

}  // extern "C"
