// Rows of a table by token, and the table's gradient (include/mtdao_ops.h).
//
// The gradient sums, for every row of the table, the rows of dy whose token it
// is.  Tokens are sorted with their places first (least significant digit first,
// stable), so each row's places lie together and in order: the
// order of every sum is fixed by the tokens alone, and nothing is added by atomics.
// Runs of more than kRun places are summed in pieces of kRun by groups of lanes of
// their own, and the pieces' sums in order by another launch.

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
constexpr int kSumE = 4;  // elements of a lane's vector of the gradient: 16 bytes of fp32, so that a wave stores whole lines at once

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

// Elements of a thread's vector: 16 bytes of the wider type.
template <typename T, typename OT>
constexpr int kE = 16 / (int)(sizeof(T) > sizeof(OT) ? sizeof(T) : sizeof(OT));

// A vector a thread.  Bound by HBM (16384 x 2048 bf16 over tensors of which the 256 MB cache holds some 18 us), few
// tokens by the launch and three dependent reads.
template <typename T, typename OT>
__global__ __launch_bounds__(kThreads) void k_embedding(Lookup a) {
  constexpr int N = kE<T, OT>;
  const int64_t at = this_group() * kThreads + threadIdx.x, i = at / a.vectors;
  if (i >= a.n) return;
  const int64_t e = (at - i * a.vectors) * N, id = id_of(a.tokens, a.wide, i);
  const int n = a.d - e > N ? N : (int)(a.d - e);
  float v[N];
#pragma unroll
  for (int t = 0; t < N; ++t) v[t] = id < 0 ? 0.0f : NAN;
  if (id >= 0 && id < a.rows) {
    load_some<N>(reinterpret_cast<const T*>(a.table) + id * a.ld + e, n, v);
#pragma unroll
    for (int t = 0; t < N; ++t) v[t] *= a.scale;
  }
  store_some<N>(reinterpret_cast<OT*>(a.out) + i * a.ld_out + e, n, v);
}

// --------------------------------------------------------------------- sort

struct Sort {
  const void* tokens;      // first pass: keys are made of them
  const uint32_t *key, *place;
  uint32_t *key_out, *place_out;
  uint32_t* counts;        // [tiles][kDigit]
  int64_t n, rows, tile;
  int32_t wide, shift, first, tiles;
  uint32_t *run_first, *run_last;  // where the places of rows that come begin and end (NULL: not wanted)
};
// The key of a token: its row, or, where it has none, the number of rows.
__device__ __forceinline__ uint32_t key_of(const Sort& a, int64_t i) {
  if (!a.first) return a.key[i];
  const int64_t id = id_of(a.tokens, a.wide, i);
  return (uint32_t)(id < 0 || id >= a.rows ? a.rows : id);
}

// The lanes whose digit is this lane's, of the live ones.
template <int BITS>
__device__ __forceinline__ uint64_t same_digit(uint32_t digit, bool live) {
  uint64_t same = __ballot(live);
#pragma unroll
  for (int b = 0; b < BITS; ++b) {
    const uint64_t set = __ballot(digit >> b & 1);
    same &= digit >> b & 1 ? set : ~set;
  }
  return same;
}
__device__ __forceinline__ int below(uint64_t lanes) { return __popcll(lanes & ((uint64_t(1) << (threadIdx.x % 64)) - 1)); }

// A run of sorted places begins or ends at place i.
__device__ __forceinline__ void mark_runs(const Sort& a, uint32_t key, uint32_t before, uint32_t after, int64_t i) {
  if (key >= a.rows) return;
  if (i == 0 || before != key) a.run_first[key] = (uint32_t)i;
  if (i == a.n - 1 || after != key) a.run_last[key] = (uint32_t)i + 1;
}

// Up to kSmall tokens of a table of fewer than 2^(32 - kPlaceBits) rows: all in the LDS of one workgroup, a word each
// (its row above its place), in two passes of BITS bits.  A wave has a run of the places, whose digits it
// counts for itself.  Bound by one CU's instructions: 2048 tokens 9 us, 16384 would take 31 us.  (The whole gradient onto 50304 rows of 64
// columns, so / by passes as below: 64 tokens 11.0 / 12.9 us, 2048 20.1 / 22.8.)
constexpr int kPlaceBits = 14, kSmall = 2048, kSmallThreads = 1024, kSmallWaves = kSmallThreads / 64, kSmallItems = kSmall / kSmallThreads;
template <int BITS>
__global__ __launch_bounds__(kSmallThreads) void k_embedding_sort(Sort a) {
  constexpr int kBins = 1 << BITS;
  extern __shared__ uint32_t words[];  // [2][n up to a multiple of 1024], [waves][kBins]
  const int tid = (int)threadIdx.x, lane = tid % 64, wave = tid / 64, n = (int)a.n, each = (n + kSmallThreads - 1) / kSmallThreads;
  const int room = each * kSmallThreads, base = wave * each * 64 + lane;
  uint32_t *buf[2] = {words, words + room}, *bins = words + 2 * room;
  for (int i = tid; i < n; i += kSmallThreads) buf[0][i] = key_of(a, i) << kPlaceBits | (uint32_t)i;
#pragma unroll
  for (int pass = 0; pass < 2; ++pass) {
    const uint32_t *from = buf[pass];
    uint32_t *to = buf[pass ^ 1], *sums = to;  // (free until items move)
    const int shift = kPlaceBits + pass * BITS;
    for (int i = tid; i < kSmallWaves * kBins; i += kSmallThreads) bins[i] = 0;
    __syncthreads();
    uint32_t* mine = bins + wave * kBins;
    uint32_t item[kSmallItems];
    uint16_t rank[kSmallItems];
#pragma unroll
    for (int r = 0; r < kSmallItems; ++r) {
      if (r < each) {
        const int i = base + r * 64;
        const bool live = i < n;
        item[r] = live ? from[i] : 0;
        const uint32_t digit = item[r] >> shift & (kBins - 1);
        const uint64_t same = same_digit<BITS>(digit, live);
        const uint32_t before = live ? mine[digit] : 0;
        rank[r] = (uint16_t)(before + below(same));
        lanes_done();
        if (live && below(same) == 0) mine[digit] = before + (uint32_t)__popcll(same);
        lanes_done();
      }
    }
    __syncthreads();
    // where each wave's items of a digit go: digits before, then waves before
    uint32_t all = 0;
    if (tid < kBins) {
#pragma unroll
      for (int w = 0; w < kSmallWaves; ++w) {
        const uint32_t c = bins[w * kBins + tid];
        bins[w * kBins + tid] = all;
        all += c;
      }
    }
    uint32_t upto = all;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const uint32_t v = __shfl_up(upto, o);
      if (lane >= o) upto += v;
    }
    if (tid < kBins && lane == 63) sums[wave] = upto;
    __syncthreads();
    if (tid < kBins) {
      uint32_t start = upto - all;
      for (int w = 0; w < wave; ++w) start += sums[w];
#pragma unroll
      for (int w = 0; w < kSmallWaves; ++w) bins[w * kBins + tid] += start;
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < kSmallItems; ++r)
      if (r < each && base + r * 64 < n) to[mine[item[r] >> shift & (kBins - 1)] + rank[r]] = item[r];
    __syncthreads();
  }
  for (int i = tid; i < n; i += kSmallThreads) {
    const uint32_t key = buf[0][i] >> kPlaceBits;
    a.key_out[i] = key;
    a.place_out[i] = buf[0][i] & ((1 << kPlaceBits) - 1);
    if (a.run_first) mark_runs(a, key, i > 0 ? buf[0][i - 1] >> kPlaceBits : 0, i + 1 < n ? buf[0][i + 1] >> kPlaceBits : 0, i);
  }
}

// More of them, up to kMiddle: a launch for each digit of BITS bits, a workgroup for each 1024 places.  Every
// workgroup counts all digits, those of the places before its own apart, rather than wait
// for another launch to do it: 16384 tokens 10 to 13 us a pass, most of it counting (a digit that many tokens share
// is counted one after the other).  That grows with the square of the places.  The whole gradient in us, by passes / by tiles
// as below, of 64 columns and 50304 rows, tokens as words come and evenly drawn: 4096 29 / 36 and 24 / 31, 16384 42 / 39 and
// 31 / 33 (of 200000 rows, a tile's pass more: 47 / 52 and 41 / 49), 24576 50 / 42 and 37 / 34, 65536 102 / 61 and 68 / 42.
constexpr int kMiddle = 16384;
template <int BITS>
__global__ __launch_bounds__(kSmallThreads) void k_embedding_pass(Sort a) {
  constexpr int kBins = 1 << BITS, kApart = 4;  // counters of a digit: one for each four waves
  __shared__ uint32_t before[kApart][kBins], rest[kApart][kBins], of_wave[kSmallWaves][kBins], start[kBins], sums[kSmallWaves];
  const int tid = (int)threadIdx.x, lane = tid % 64, wave = tid / 64, n = (int)a.n, base = (int)blockIdx.x * kSmallThreads;
  for (int i = tid; i < kApart * kBins; i += kSmallThreads) (&before[0][0])[i] = (&rest[0][0])[i] = 0;
  for (int i = tid; i < kSmallWaves * kBins; i += kSmallThreads) (&of_wave[0][0])[i] = 0;
  __syncthreads();
  const int at = base + tid;
  const bool live = at < n;
  const uint32_t key = live ? key_of(a, at) : 0, digit = key >> a.shift & (kBins - 1);
  const uint32_t place = live ? (a.first ? (uint32_t)at : a.place[at]) : 0;
#pragma unroll 8
  for (int i = tid; i < n; i += kSmallThreads) {
    const uint32_t d = key_of(a, i) >> a.shift & (kBins - 1);
    atomicAdd(i < base ? &before[wave % kApart][d] : &rest[wave % kApart][d], 1u);
  }
  const uint64_t same = same_digit<BITS>(digit, live);
  if (live && below(same) == 0) of_wave[wave][digit] = (uint32_t)__popcll(same);
  __syncthreads();
  uint32_t mine = 0, all = 0, upto;
  if (tid < kBins) {
#pragma unroll
    for (int w = 0; w < kApart; ++w) {
      mine += before[w][tid];
      all += rest[w][tid];
    }
    all += mine;
  }
  upto = all;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const uint32_t v = __shfl_up(upto, o);
    if (lane >= o) upto += v;
  }
  if (lane == 63) sums[wave] = upto;
  __syncthreads();
  if (tid < kBins) {
    for (int w = 0; w < wave; ++w) upto += sums[w];
    start[tid] = upto - all + mine;
  }
  __syncthreads();
  if (!live) return;
  uint32_t to = start[digit] + (uint32_t)below(same);
  for (int w = 0; w < wave; ++w) to += of_wave[w][digit];
  a.key_out[to] = key;
  a.place_out[to] = place;
}

// More still: tiles of places, eight bits a pass.
constexpr int kDigit = 256;                      // values of a digit
constexpr int kLeastTile = 1024, kMostTiles = 256;  // places of a workgroup; tiles, which every workgroup of the second launch sums up

__global__ __launch_bounds__(kThreads) void k_embedding_count(Sort a) {
  __shared__ uint32_t bins[kDigit];
  bins[threadIdx.x] = 0;
  __syncthreads();
  const int64_t base = (int64_t)blockIdx.x * a.tile, end = base + a.tile < a.n ? base + a.tile : a.n;
  for (int64_t i = base + threadIdx.x; i < end; i += kThreads) atomicAdd(&bins[key_of(a, i) >> a.shift & (kDigit - 1)], 1u);
  __syncthreads();
  a.counts[(int64_t)blockIdx.x * kDigit + threadIdx.x] = bins[threadIdx.x];
}

// Places of a tile to where their digit begins, in their order.
__global__ __launch_bounds__(kThreads) void k_embedding_move(Sort a) {
  constexpr int kWaves = kThreads / 64;
  __shared__ uint32_t start[kDigit], sums[kWaves];
  __shared__ uint32_t of_wave[kWaves][kDigit];
  const int tid = threadIdx.x, lane = tid % 64, wave = tid / 64;
  uint32_t before = 0, all = 0;
#pragma unroll 8
  for (int t = 0; t < a.tiles; ++t) {
    const uint32_t c = a.counts[(int64_t)t * kDigit + tid];
    before += t < (int)blockIdx.x ? c : 0;
    all += c;
  }
  uint32_t upto = all;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const uint32_t v = __shfl_up(upto, o);
    if (lane >= o) upto += v;
  }
  if (lane == 63) sums[wave] = upto;
  __syncthreads();
  for (int w = 0; w < wave; ++w) upto += sums[w];
  start[tid] = upto - all + before;
  const int64_t base = (int64_t)blockIdx.x * a.tile, end = base + a.tile < a.n ? base + a.tile : a.n;
  for (int64_t from = base; from < end; from += kThreads) {
    const int64_t i = from + tid;
    const bool live = i < end;
    const uint32_t key = live ? key_of(a, i) : 0, digit = key >> a.shift & (kDigit - 1);
    const uint32_t place = live ? (a.first ? (uint32_t)i : a.place[i]) : 0;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kWaves; ++w) of_wave[w][tid] = 0;
    __syncthreads();
    const uint64_t same = same_digit<8>(digit, live);
    const int rank = below(same);
    if (live && rank == 0) of_wave[wave][digit] = (uint32_t)__popcll(same);
    __syncthreads();
    if (live) {
      uint32_t to = start[digit] + (uint32_t)rank;
      for (int w = 0; w < wave; ++w) to += of_wave[w][digit];
      a.key_out[to] = key;
      a.place_out[to] = place;
    }
    __syncthreads();
    uint32_t more = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) more += of_wave[w][tid];
    start[tid] += more;
  }
}

// The runs of the rows that come, from sorted keys.
__global__ __launch_bounds__(kThreads) void k_embedding_marks(Sort a) {
  const int64_t i = this_group() * kThreads + threadIdx.x;
  if (i < a.n) mark_runs(a, a.key[i], i > 0 ? a.key[i - 1] : 0, i + 1 < a.n ? a.key[i + 1] : 0, i);
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

// Places that a lane adds up, eight in flight.  Pieces of 16 / 32 / 64, the whole gradient in us: 16384 x 2048 into a new one of 50304 rows
// 134 / 121 / 119, of 8192 rows 79 / 70 / 76, of 256 rows 48 / 45 / 55; 16384 places of one token x 768 173 / 121 / 99; 4096 x 1024 onto 16 rows
// 23 / 26 / 37, 1999 x 768 onto 50304 21 / 25 / 32.
constexpr int kRun = 32;
constexpr int kSlot = kRun / 2;
// Lanes that work on the same places, a vector of the columns each.  (Groups of 64: the whole gradient, 16384 places, 50304 rows
// of 64 columns 44.5 us in place of 41.5, of 68 to 2048 the same within 1%.)
constexpr int kGroup = 16;

struct Sums {
  const uint32_t *key, *place, *first, *last;  // first and last: of a row's places
  const void* dy;
  float *dw, *pieces;   // pieces: [slots][d]
  int64_t n, rows, d, ld_dy, ld_dw;
  int64_t slots, chunks;  // chunks of a row: a vector for each of a group of lanes
  float scale;
  int32_t onto;
};

// Adds rows of dy: the group's lanes fetch their places together, and eight rows are in flight.
template <typename T>
__device__ __forceinline__ void add_rows(const Sums& a, int64_t from, int64_t to, int64_t e, int n, float (&sum)[kSumE]) {
  const T* dy = reinterpret_cast<const T*>(a.dy) + e;
  const int lane = (int)threadIdx.x % 64, in = lane % kGroup;
  for (; from < to; from += kGroup) {
    const int count = to - from < kGroup ? (int)(to - from) : kGroup;
    const uint32_t mine = in < count ? a.place[from + in] : 0;
    for (int i = 0; i < count; i += 8) {
      float v[8][kSumE];
#pragma unroll
      for (int t = 0; t < 8; ++t) {
        const uint32_t place = (uint32_t)__shfl((int)mine, lane - in + (i + t) % kGroup);
        if (i + t < count) load_some<kSumE>(dy + (int64_t)place * a.ld_dy, n, v[t]);
      }
#pragma unroll
      for (int t = 0; t < 8; ++t)
        if (i + t < count) {
#pragma unroll
          for (int k = 0; k < kSumE; ++k) sum[k] += v[t][k];
        }
    }
  }
}

// sum to row `row` of dw.
__device__ __forceinline__ void store_sum(const Sums& a, int64_t row, int64_t e, int n, const float (&sum)[kSumE]) {
  float* dw = a.dw + row * a.ld_dw + e;
  float o[kSumE] = {};
  if (a.onto) load_some<kSumE>(dw, n, o);
#pragma unroll
  for (int t = 0; t < kSumE; ++t) o[t] = a.onto ? fmaf(sum[t], a.scale, o[t]) : sum[t] * a.scale;
  if (n > 0) store_some<kSumE, true>(dw, n, o);
}

// What a slot holds: a run of c > kRun places from place s on has the slots
// s / kSlot + j of its pieces j.  The last place of slot q's kSlot places belongs to
// the run that the slot is of, if any, and no two runs share one, since c / kSlot >=
// c / kRun rounded up.
struct Piece {
  int64_t row, s, c, j;
};
__device__ __forceinline__ bool piece_of(const Sums& a, int64_t slot, Piece& p) {
  const int64_t probe = slot * kSlot + kSlot - 1;
  if (probe >= a.n) return false;
  p.row = a.key[probe];
  if (p.row >= a.rows) return false;
  p.s = a.first[p.row];
  p.c = (int64_t)a.last[p.row] - p.s;
  p.j = slot - p.s / kSlot;
  return p.c > kRun && p.j * kRun < p.c;
}

// Pieces of long runs (first, as they take longest), and rows of runs that have none: a job for
// each row of the table, or for each place.  Bound by HBM's writes where the gradient is new: 50304 x 2048
// from 16384 tokens 74 us, 6.5 TB/s.  (Clearing it in the launch that sorts, and then only the rows that come: 132 us in all
// in place of 104.)
template <typename T>
__global__ __launch_bounds__(kThreads) void k_embedding_sums(Sums a) {
  const int64_t job = this_group() * (kThreads / kGroup) + (int)threadIdx.x / kGroup, at = job / a.chunks;
  const int64_t e = ((job - at * a.chunks) * kGroup + (int)threadIdx.x % kGroup) * kSumE;
  const int n = a.d - e > kSumE ? kSumE : a.d > e ? (int)(a.d - e) : 0;
  float sum[kSumE] = {};
  if (at < a.slots) {
    Piece p;
    if (!piece_of(a, at, p)) return;
    const int64_t from = p.s + p.j * kRun, end = p.s + p.c;
    add_rows<T>(a, from, from + kRun < end ? from + kRun : end, e, n, sum);
    if (n > 0) store_some<kSumE>(a.pieces + at * a.d + e, n, sum);
    return;
  }
  int64_t row = at - a.slots;
  if (a.onto) {  // a job for each place: the first one of a run has the run
    if (row >= a.n) return;
    const int64_t place = row;
    row = a.key[place];
    if (row >= a.rows || (place > 0 && a.key[place - 1] == row)) return;
  } else if (row >= a.rows) {
    return;
  }
  const int64_t s = a.first[row], c = (int64_t)a.last[row] - s;
  if (c > kRun) return;
  add_rows<T>(a, s, s + c, e, n, sum);
  store_sum(a, row, e, n, sum);
}

// Rows of long runs from their pieces, eight in flight.
__global__ __launch_bounds__(kThreads) void k_embedding_join(Sums a) {
  const int64_t vectors = (a.d + kSumE - 1) / kSumE, job = this_group() * kThreads + threadIdx.x, slot = job / vectors;
  Piece p;
  if (slot >= a.slots || !piece_of(a, slot, p) || p.j != 0) return;
  const int64_t e = (job - slot * vectors) * kSumE, pieces = (p.c + kRun - 1) / kRun;
  const int n = a.d - e > kSumE ? kSumE : (int)(a.d - e);
  float sum[kSumE] = {};
  for (int64_t j = 0; j < pieces; j += 8) {
    float v[8][kSumE];
#pragma unroll
    for (int t = 0; t < 8; ++t)
      if (j + t < pieces) load_some<kSumE>(a.pieces + (slot + j + t) * a.d + e, n, v[t]);
#pragma unroll
    for (int t = 0; t < 8; ++t)
      if (j + t < pieces) {
#pragma unroll
        for (int k = 0; k < kSumE; ++k) sum[k] += v[t][k];
      }
  }
  store_sum(a, p.row, e, n, sum);
}

// --------------------------------------------------------------------- host

int64_t over(int64_t n, int64_t m) { return (n + m - 1) / m; }

int32_t check_sizes(int64_t n, int64_t rows, int64_t d, std::string* e) {
  if (n < 0 || n > (INT64_C(1) << 30)) return fail(e, MTDAO_ERR_INVALID_ARG, "%lld tokens: 0..2^30", (long long)n);
  if (rows < 0 || rows > (INT64_C(1) << 30)) return fail(e, MTDAO_ERR_INVALID_ARG, "rows %lld: 0..2^30", (long long)rows);
  if (d < 1 || d > (INT64_C(1) << 20)) return fail(e, MTDAO_ERR_INVALID_ARG, "d %lld: 1..2^20", (long long)d);
  // (workgroups of a launch)
  if (over((n + rows) * over(d, kSumE), kThreads / 64) > kGridMost)
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
  size_t key[2], place[2], counts, first, last, pieces, bytes;
  int64_t tile, tiles, slots;
};
Layout layout_of(int64_t n, int64_t rows, int64_t d) {
  Layout l;
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t here = at;
    at += up256(bytes);
    return here;
  };
  l.tile = std::max<int64_t>(kLeastTile, over(over(n, kMostTiles), kThreads) * kThreads);
  l.tiles = over(n, l.tile);
  l.slots = n / kSlot + 1;
  for (int i = 0; i < 2; ++i) {
    l.key[i] = take((size_t)n * 4);
    l.place[i] = take((size_t)n * 4);
  }
  l.counts = take((size_t)l.tiles * kDigit * 4);
  l.first = take((size_t)(rows + 1) * 4);
  l.last = take((size_t)rows * 4);
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
  hipStream_t st = reinterpret_cast<hipStream_t>(hip_stream);
  RoctxRange range("mtdao_embedding %lld x %lld", (long long)n_tokens, (long long)d);
  auto go = [&](auto t, auto o) {
    using T = decltype(t);
    using OT = decltype(o);
    const Lookup a = {tokens, table, out, n_tokens, rows, d, ld, ld_out, over(d, kE<T, OT>), token_bits == 64, scale};
    hipLaunchKernelGGL((k_embedding<T, OT>), grid_of(over(n_tokens * a.vectors, kThreads)), dim3(kThreads), 0, st, a);
  };
  if (table_dtype == MTDAO_F32 && out_dtype == MTDAO_F32) go(float{}, float{});
  else if (table_dtype == MTDAO_F32) go(float{}, bf16_t{});
  else if (out_dtype == MTDAO_F32) go(bf16_t{}, float{});
  else go(bf16_t{}, bf16_t{});
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
  Sort sort = {tokens, words(l.key[1]), words(l.place[1]), words(l.key[0]), words(l.place[0]), words(l.counts), n_tokens, rows, l.tile,
               token_bits == 64, 0, 1, (int32_t)l.tiles, nullptr, nullptr};
  // Added onto a gradient, only the rows that come count: their runs are found by place.  A new one has a job for each row.
  if (accumulate) {
    sort.run_first = words(l.first);
    sort.run_last = words(l.last);
  }
  if (n_tokens > 0 && n_tokens <= kSmall && bits <= 32 - kPlaceBits) {
    const int64_t room = over(n_tokens, kSmallThreads) * kSmallThreads;
    auto lds = [&](int bins) { return (size_t)(2 * room + kSmallWaves * bins) * 4; };
    if (bits <= 16) hipLaunchKernelGGL(k_embedding_sort<8>, dim3(1), dim3(kSmallThreads), lds(256), st, sort);
    else hipLaunchKernelGGL(k_embedding_sort<9>, dim3(1), dim3(kSmallThreads), lds(512), st, sort);
  } else if (n_tokens > 0) {
    const bool middle = n_tokens <= kMiddle;
    const int digit = middle && over(bits, 9) < over(bits, 8) ? 9 : 8;
    for (; sort.shift < bits; sort.shift += digit, at ^= 1) {
      sort.first = sort.shift == 0;
      sort.key = words(l.key[at ^ 1]);
      sort.place = words(l.place[at ^ 1]);
      sort.key_out = words(l.key[at]);
      sort.place_out = words(l.place[at]);
      if (middle) {
        const dim3 grid((unsigned)over(n_tokens, kSmallThreads));
        if (digit == 8) hipLaunchKernelGGL(k_embedding_pass<8>, grid, dim3(kSmallThreads), 0, st, sort);
        else hipLaunchKernelGGL(k_embedding_pass<9>, grid, dim3(kSmallThreads), 0, st, sort);
      } else {
        hipLaunchKernelGGL(k_embedding_count, dim3((unsigned)l.tiles), block, 0, st, sort);
        hipLaunchKernelGGL(k_embedding_move, dim3((unsigned)l.tiles), block, 0, st, sort);
      }
    }
    at ^= 1;
    if (accumulate) {
      sort.key = words(l.key[at]);
      hipLaunchKernelGGL(k_embedding_marks, grid_of(over(n_tokens, kThreads)), block, 0, st, sort);
    }
  }
  if (!accumulate)
    hipLaunchKernelGGL(k_embedding_runs, grid_of(over(rows + 1, kThreads)), block, 0, st, words(l.key[at]), (uint32_t)n_tokens, rows, words(l.first));
  const int64_t vectors = over(d, kSumE);
  Sums s = {words(l.key[at]), words(l.place[at]), words(l.first), accumulate ? words(l.last) : words(l.first) + 1, dy, dw, reinterpret_cast<float*>(w + l.pieces), n_tokens, rows, d, ld_dy, ld_dw,
            n_tokens > kRun ? l.slots : 0, over(vectors, kGroup), scale, accumulate};
  auto go = [&](auto t) {
    using T = decltype(t);
    const int64_t jobs = (s.slots + (accumulate ? n_tokens : rows)) * s.chunks;
    hipLaunchKernelGGL(k_embedding_sums<T>, grid_of(over(jobs, kThreads / kGroup)), block, 0, st, s);
    if (s.slots > 0) hipLaunchKernelGGL(k_embedding_join, grid_of(over(s.slots * vectors, kThreads)), block, 0, st, s);
  };
  if (dy_dtype == MTDAO_BF16) go(bf16_t{});
  else go(float{});
  return hip_check(e, hipGetLastError(), "mtdao_embedding_backward launch");
}

}  // extern "C"
