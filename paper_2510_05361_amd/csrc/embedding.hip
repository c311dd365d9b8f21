// Rows of a table by token, and the table's gradient (include/mtdao_ops.h).
//
// The gradient sums, for every row of the table, the rows of dy whose token it
// is.  Tokens are sorted with their places first (least significant digit first,
// eight bits at once, stable), so each row's places lie together and in order: the
// order of every sum is fixed by the tokens alone, and nothing is added by atomics.
// Runs of more than kRun places are summed in pieces of kRun by workgroups of
// their own, and the pieces' sums in order.

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
constexpr int kE = 8;  // elements of a thread's vector

__device__ __forceinline__ int64_t id_of(const void* ids, int32_t wide, int64_t i) {
  return wide ? reinterpret_cast<const int64_t*>(ids)[i] : (int64_t) reinterpret_cast<const int32_t*>(ids)[i];
}
__device__ __forceinline__ int64_t this_group() { return (int64_t)blockIdx.y * gridDim.x + blockIdx.x; }

// ------------------------------------------------------------------- lookup

struct Lookup {
  const void* tokens;
  const void* table;
  void* out;
  int64_t n, rows, d, ld, ld_out;
  int64_t vectors;  // of a row
  int32_t wide;
  float scale;
};

template <typename T, typename OT>
__global__ __launch_bounds__(kThreads) void k_embedding(Lookup a) {
  const int64_t at = this_group() * kThreads + threadIdx.x, i = at / a.vectors;
  if (i >= a.n) return;
  const int64_t e = (at - i * a.vectors) * kE, id = id_of(a.tokens, a.wide, i);
  const int n = a.d - e > kE ? kE : (int)(a.d - e);
  float v[kE];
#pragma unroll
  for (int t = 0; t < kE; ++t) v[t] = id < 0 ? 0.0f : NAN;
  if (id >= 0 && id < a.rows) {
    load_some<kE>(reinterpret_cast<const T*>(a.table) + id * a.ld + e, n, v);
#pragma unroll
    for (int t = 0; t < kE; ++t) v[t] *= a.scale;
  }
  store_some<kE>(reinterpret_cast<OT*>(a.out) + i * a.ld_out + e, n, v);
}

// --------------------------------------------------------------------- sort

constexpr int kDigit = 256;       // values of a digit
constexpr int kSortTile = 4096;   // places of a workgroup

struct Sort {
  const void* tokens;      // first pass: keys are made of them
  const uint32_t *key, *place;
  uint32_t *key_out, *place_out;
  uint32_t* counts;        // [tiles][kDigit]
  int64_t n, rows;
  int32_t wide, shift, first, tiles;
};
// The key of a token: its row, or, where it has none, the number of rows.
__device__ __forceinline__ uint32_t key_of(const Sort& a, int64_t i) {
  if (!a.first) return a.key[i];
  const int64_t id = id_of(a.tokens, a.wide, i);
  return (uint32_t)(id < 0 || id >= a.rows ? a.rows : id);
}

__global__ __launch_bounds__(kThreads) void k_embedding_count(Sort a) {
  __shared__ uint32_t bins[kDigit];
  bins[threadIdx.x] = 0;
  __syncthreads();
  const int64_t base = (int64_t)blockIdx.x * kSortTile;
  for (int t = threadIdx.x; t < kSortTile && base + t < a.n; t += kThreads) atomicAdd(&bins[key_of(a, base + t) >> a.shift & (kDigit - 1)], 1u);
  __syncthreads();
  a.counts[(int64_t)blockIdx.x * kDigit + threadIdx.x] = bins[threadIdx.x];
}

// Places of a tile to where their digit begins, in their order.
__global__ __launch_bounds__(kThreads) void k_embedding_move(Sort a) {
  constexpr int kWaves = kThreads / 64;
  __shared__ uint32_t start[kDigit], sums[kDigit];
  __shared__ uint32_t of_wave[kWaves][kDigit];
  const int tid = threadIdx.x, lane = tid % 64, wave = tid / 64;
  uint32_t before = 0, all = 0;
  for (int t = 0; t < a.tiles; ++t) {
    const uint32_t c = a.counts[(int64_t)t * kDigit + tid];
    before += t < (int)blockIdx.x ? c : 0;
    all += c;
  }
  sums[tid] = all;
  __syncthreads();
  for (int o = 1; o < kDigit; o <<= 1) {
    const uint32_t v = tid >= o ? sums[tid - o] : 0;
    __syncthreads();
    sums[tid] += v;
    __syncthreads();
  }
  start[tid] = sums[tid] - all + before;
  const int64_t base = (int64_t)blockIdx.x * kSortTile;
  for (int from = 0; from < kSortTile; from += kThreads) {
    const int64_t i = base + from + tid;
    const bool live = i < a.n;
    const uint32_t key = live ? key_of(a, i) : 0, digit = key >> a.shift & (kDigit - 1);
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kWaves; ++w) of_wave[w][tid] = 0;
    __syncthreads();
    uint64_t same = __ballot(live);
#pragma unroll
    for (int b = 0; b < 8; ++b) {
      const uint64_t set = __ballot(digit >> b & 1);
      same &= digit >> b & 1 ? set : ~set;
    }
    const int rank = __popcll(same & ((uint64_t(1) << lane) - 1));
    if (live && rank == 0) of_wave[wave][digit] = (uint32_t)__popcll(same);
    __syncthreads();
    if (live) {
      uint32_t to = start[digit] + (uint32_t)rank;
      for (int w = 0; w < wave; ++w) to += of_wave[w][digit];
      a.key_out[to] = key;
      a.place_out[to] = a.first ? (uint32_t)i : a.place[i];
    }
    __syncthreads();
    uint32_t more = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) more += of_wave[w][tid];
    start[tid] += more;
  }
}

// Where each row's places begin: first[row], for rows 0..rows, by halving.
__global__ __launch_bounds__(kThreads) void k_embedding_runs(const uint32_t* key, uint32_t n, int64_t rows, uint32_t* first) {
  const int64_t row = this_group() * kThreads + threadIdx.x;
  if (row > rows) return;
  uint32_t from = 0, to = n;
  while (from < to) {
    const uint32_t mid = (from + to) / 2;
    if (key[mid] < (uint32_t)row) from = mid + 1;
    else to = mid;
  }
  first[row] = from;
}

// --------------------------------------------------------------------- sums

constexpr int kRun = 64;       // places that one thread adds up
constexpr int kSlot = kRun / 2;

struct Sums {
  const uint32_t *key, *place, *first;
  const void* dy;
  float *dw, *pieces;   // pieces: [slots][d]
  int64_t n, rows, d, ld_dy, ld_dw, vectors;
  float scale;
  int32_t onto;
};

template <typename T>
__device__ __forceinline__ void add_rows(const Sums& a, int64_t from, int64_t to, int64_t e, int n, float (&sum)[kE]) {
  const T* dy = reinterpret_cast<const T*>(a.dy) + e;
#pragma unroll 4
  for (int64_t i = from; i < to; ++i) {
    float v[kE];
    load_some<kE>(dy + (int64_t)a.place[i] * a.ld_dy, n, v);
#pragma unroll
    for (int t = 0; t < kE; ++t) sum[t] += v[t];
  }
}

// The pieces of long runs.  A run of c > kRun places from place s on has the slots
// s / kSlot + j of its pieces j: the place 31 of slot q's kSlot places belongs to
// the run that the slot is of, if any, and no two runs share one, since c / kSlot >=
// c / kRun rounded up.
template <typename T>
__global__ __launch_bounds__(kThreads) void k_embedding_pieces(Sums a) {
  const int64_t at = this_group() * kThreads + threadIdx.x, slot = at / a.vectors, probe = slot * kSlot + kSlot - 1;
  if (probe >= a.n) return;
  const uint32_t row = a.key[probe];
  if (row >= a.rows) return;
  const int64_t s = a.first[row], c = (int64_t)a.first[row + 1] - s, j = slot - s / kSlot;
  if (c <= kRun || j * kRun >= c) return;
  const int64_t e = (at - slot * a.vectors) * kE;
  const int n = a.d - e > kE ? kE : (int)(a.d - e);
  float sum[kE] = {};
  add_rows<T>(a, s + j * kRun, s + (j * kRun + kRun < c ? j * kRun + kRun : c), e, n, sum);
  store_some<kE>(a.pieces + slot * a.d + e, n, sum);
}

template <typename T>
__global__ __launch_bounds__(kThreads) void k_embedding_sums(Sums a) {
  const int64_t at = this_group() * kThreads + threadIdx.x, row = at / a.vectors;
  if (row >= a.rows) return;
  const int64_t e = (at - row * a.vectors) * kE, s = a.first[row], c = (int64_t)a.first[row + 1] - s;
  const int n = a.d - e > kE ? kE : (int)(a.d - e);
  float* dw = a.dw + row * a.ld_dw + e;
  if (c == 0 && a.onto) return;
  float sum[kE] = {};
  if (c <= kRun) {
    add_rows<T>(a, s, s + c, e, n, sum);
  } else {
    const float* piece = a.pieces + s / kSlot * a.d + e;
    for (int64_t j = 0; j * kRun < c; ++j) {
      float v[kE];
      load_some<kE>(piece + j * a.d, n, v);
#pragma unroll
      for (int t = 0; t < kE; ++t) sum[t] += v[t];
    }
  }
  float o[kE] = {};
  if (a.onto) load_some<kE>(dw, n, o);
#pragma unroll
  for (int t = 0; t < kE; ++t) o[t] = a.onto ? fmaf(sum[t], a.scale, o[t]) : sum[t] * a.scale;
  store_some<kE>(dw, n, o);
}

// --------------------------------------------------------------------- host

size_t up256(size_t n) { return (n + 255) / 256 * 256; }
int64_t esize(int32_t dt) { return dt == MTDAO_BF16 ? 2 : 4; }
int64_t over(int64_t n, int64_t m) { return (n + m - 1) / m; }

int32_t check_sizes(int64_t n, int64_t rows, int64_t d, std::string* e) {
  if (n < 0 || n > (INT64_C(1) << 30)) return fail(e, MTDAO_ERR_INVALID_ARG, "%lld tokens: 0..2^30", (long long)n);
  if (rows < 0 || rows > (INT64_C(1) << 30)) return fail(e, MTDAO_ERR_INVALID_ARG, "rows %lld: 0..2^30", (long long)rows);
  if (d < 1 || d > (INT64_C(1) << 20)) return fail(e, MTDAO_ERR_INVALID_ARG, "d %lld: 1..2^20", (long long)d);
  // (workgroups of a launch)
  if (over(std::max(n, rows) * over(d, kE), kThreads) > kGridMost)
    return fail(e, MTDAO_ERR_INVALID_ARG, "the operands exceed the largest launch");
  return MTDAO_OK;
}
int32_t check_tokens(const void* tokens, int32_t bits, int64_t n, std::string* e) {
  if (bits != 32 && bits != 64) return fail(e, MTDAO_ERR_INVALID_ARG, "token_bits %d is not 32 or 64", bits);
  if (n > 0 && !tokens) return fail(e, MTDAO_ERR_INVALID_ARG, "tokens is NULL");
  if (!aligned_to(tokens, (uintptr_t)bits / 8)) return fail(e, MTDAO_ERR_ALIGN, "tokens are not aligned to their element");
  return MTDAO_OK;
}
int32_t check_rows(const void* x, int32_t dtype, int64_t rows, int64_t d, int64_t ld, const char* name, std::string* e) {
  if (dtype != MTDAO_F32 && dtype != MTDAO_BF16) return fail(e, MTDAO_ERR_INVALID_ARG, "the type of %s must be F32(0) or BF16(1)", name);
  if (rows == 0) return MTDAO_OK;
  if (ld < d || ld > (INT64_C(1) << 42) / rows)
    return fail(e, MTDAO_ERR_INVALID_ARG, "row stride %lld of %s is below its columns or exceeds 2^42 elements in all", (long long)ld, name);
  if (!x) return fail(e, MTDAO_ERR_INVALID_ARG, "%s is NULL", name);
  if (!aligned_to(x, (uintptr_t)esize(dtype))) return fail(e, MTDAO_ERR_ALIGN, "%s is not aligned to its element", name);
  return MTDAO_OK;
}
int64_t extent(int64_t rows, int64_t d, int64_t ld, int64_t es) { return rows > 0 ? ((rows - 1) * ld + d) * es : 0; }

struct Layout {
  size_t key[2], place[2], counts, first, pieces, bytes;
  int64_t tiles, slots;
};
Layout layout_of(int64_t n, int64_t rows, int64_t d) {
  Layout l;
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t here = at;
    at += up256(bytes);
    return here;
  };
  l.tiles = over(n, kSortTile);
  l.slots = n / kSlot + 1;
  for (int i = 0; i < 2; ++i) {
    l.key[i] = take((size_t)n * 4);
    l.place[i] = take((size_t)n * 4);
  }
  l.counts = take((size_t)l.tiles * kDigit * 4);
  l.first = take((size_t)(rows + 1) * 4);
  l.pieces = take((size_t)l.slots * d * 4);
  l.bytes = at;
  return l;
}

}  // namespace

extern "C" {

int32_t mtdao_embedding(const void* tokens, int32_t token_bits, int64_t n_tokens, const void* table, int32_t table_dtype, int64_t rows, int64_t d,
                        int64_t ld, float scale, void* out, int32_t out_dtype, int64_t ld_out, void* hip_stream) {
  std::string* e = &g_err;
  int32_t r = check_sizes(n_tokens, rows, d, e);
  if (r == MTDAO_OK) r = check_tokens(tokens, token_bits, n_tokens, e);
  if (r == MTDAO_OK) r = check_rows(table, table_dtype, rows, d, ld, "table", e);
  if (r == MTDAO_OK) r = check_rows(out, out_dtype, n_tokens, d, ld_out, "out", e);
  if (r != MTDAO_OK) return r;
  if (!std::isfinite(scale)) return fail(e, MTDAO_ERR_INVALID_ARG, "scale is not finite");
  if (n_tokens == 0) return MTDAO_OK;
  const int64_t to = extent(n_tokens, d, ld_out, esize(out_dtype));
  if (overlap(out, to, table, extent(rows, d, ld, esize(table_dtype))) || overlap(out, to, tokens, n_tokens * token_bits / 8))
    return fail(e, MTDAO_ERR_INVALID_ARG, "out overlaps table or tokens");
  const Lookup a = {tokens, table, out, n_tokens, rows, d, ld, ld_out, over(d, kE), token_bits == 64, scale};
  hipStream_t st = reinterpret_cast<hipStream_t>(hip_stream);
  RoctxRange range("mtdao_embedding %lld x %lld", (long long)n_tokens, (long long)d);
  const dim3 grid = grid_of(over(n_tokens * a.vectors, kThreads)), block(kThreads);
  if (table_dtype == MTDAO_F32 && out_dtype == MTDAO_F32) hipLaunchKernelGGL((k_embedding<float, float>), grid, block, 0, st, a);
  else if (table_dtype == MTDAO_F32) hipLaunchKernelGGL((k_embedding<float, bf16_t>), grid, block, 0, st, a);
  else if (out_dtype == MTDAO_F32) hipLaunchKernelGGL((k_embedding<bf16_t, float>), grid, block, 0, st, a);
  else hipLaunchKernelGGL((k_embedding<bf16_t, bf16_t>), grid, block, 0, st, a);
  return hip_check(e, hipGetLastError(), "mtdao_embedding launch");
}

int32_t mtdao_embedding_backward_workspace_bytes(int64_t n_tokens, int64_t rows, int64_t d, size_t* bytes) {
  const int32_t r = check_sizes(n_tokens, rows, d, &g_err);
  if (r != MTDAO_OK) return r;
  if (!bytes) return fail(&g_err, MTDAO_ERR_INVALID_ARG, "bytes is NULL");
  *bytes = layout_of(n_tokens, rows, d).bytes;
  return MTDAO_OK;
}

int32_t mtdao_embedding_backward(const void* dy, int32_t dy_dtype, int64_t ld_dy, const void* tokens, int32_t token_bits, int64_t n_tokens, float scale,
                                 float* dw, int64_t rows, int64_t d, int64_t ld_dw, int32_t accumulate, void* workspace, size_t workspace_bytes,
                                 void* hip_stream) {
  std::string* e = &g_err;
  int32_t r = check_sizes(n_tokens, rows, d, e);
  if (r == MTDAO_OK) r = check_tokens(tokens, token_bits, n_tokens, e);
  if (r == MTDAO_OK) r = check_rows(dy, dy_dtype, n_tokens, d, ld_dy, "dy", e);
  if (r == MTDAO_OK) r = check_rows(dw, MTDAO_F32, rows, d, ld_dw, "dw", e);
  if (r != MTDAO_OK) return r;
  if (!std::isfinite(scale)) return fail(e, MTDAO_ERR_INVALID_ARG, "scale is not finite");
  if (rows == 0 || (n_tokens == 0 && accumulate)) return MTDAO_OK;
  const int64_t to = extent(rows, d, ld_dw, 4);
  if (overlap(dw, to, dy, extent(n_tokens, d, ld_dy, esize(dy_dtype))) || overlap(dw, to, tokens, n_tokens * token_bits / 8))
    return fail(e, MTDAO_ERR_INVALID_ARG, "dw overlaps dy or tokens");
  const Layout l = layout_of(n_tokens, rows, d);
  if (!workspace || workspace_bytes < l.bytes)
    return fail(e, MTDAO_ERR_WORKSPACE, "workspace of %zu bytes required, %zu given", l.bytes, workspace ? workspace_bytes : (size_t)0);
  if (!aligned_to(workspace, 256)) return fail(e, MTDAO_ERR_ALIGN, "workspace is not 256-byte aligned");
  char* w = static_cast<char*>(workspace);
  hipStream_t st = reinterpret_cast<hipStream_t>(hip_stream);
  RoctxRange range("mtdao_embedding_backward %lld x %lld", (long long)n_tokens, (long long)d);
  const dim3 block(kThreads);
  auto words = [&](size_t at) { return reinterpret_cast<uint32_t*>(w + at); };
  int bits = 1;
  while (rows >> bits) ++bits;
  int at = 0;
  if (n_tokens > 0) {
    for (int shift = 0; shift < bits; shift += 8, at ^= 1) {
      const Sort s = {tokens, words(l.key[at ^ 1]), words(l.place[at ^ 1]), words(l.key[at]), words(l.place[at]), words(l.counts), n_tokens, rows,
                      token_bits == 64, shift, shift == 0, (int32_t)l.tiles};
      hipLaunchKernelGGL(k_embedding_count, dim3((unsigned)l.tiles), block, 0, st, s);
      hipLaunchKernelGGL(k_embedding_move, dim3((unsigned)l.tiles), block, 0, st, s);
    }
    at ^= 1;
  }
  hipLaunchKernelGGL(k_embedding_runs, grid_of(over(rows + 1, kThreads)), block, 0, st, words(l.key[at]), (uint32_t)n_tokens, rows, words(l.first));
  const Sums s = {words(l.key[at]), words(l.place[at]), words(l.first), dy, dw, reinterpret_cast<float*>(w + l.pieces), n_tokens, rows, d, ld_dy, ld_dw,
                  over(d, kE), scale, accumulate};
  auto go = [&](auto t) {
    using T = decltype(t);
    if (n_tokens > kRun) hipLaunchKernelGGL(k_embedding_pieces<T>, grid_of(over(l.slots * s.vectors, kThreads)), block, 0, st, s);
    hipLaunchKernelGGL(k_embedding_sums<T>, grid_of(over(rows * s.vectors, kThreads)), block, 0, st, s);
  };
  if (dy_dtype == MTDAO_BF16) go(bf16_t{});
  else go(float{});
  return hip_check(e, hipGetLastError(), "mtdao_embedding_backward launch");
}

}  // extern "C"
