// Orthogonalised updates of matrices by Newton-Schulz products, and the
// optimizer step that takes them (include/mtdao_ops.h).
//
// Numbers.  Every factor of a product is held as the sum of two fp16 numbers,
// x 2^e = hi + lo: hi is x 2^e rounded to eleven bits, lo the rest, of thirteen bits, rounded to
// eleven, so that together they are off by 2^-23 |x| at most (their root mean square is 2^-24.5 |x|; an fp32
// number is off by 2^-24 |x| at most).  A product is hi hi + hi lo + lo hi in the fp16 matrix
// instructions, each term exact and summed in fp32; lo lo, 2^-22 of the product at most as |lo| <= 2^-11 |x|,
// is left out.  That is three matrix instructions for a product of fp32's precision, at a
// sixteenth of the cost of fp32's own each.  (One bf16 term alone leaves the directions
// with small singular values, which the iteration raises 480-fold, to rounding:
// errors of 2 (Gaussian) to 40 (low rank and noise) in a hundred of the result.)
// fp16's exponents suffice because all factors are bounded: the singular values
// s of X are at most 1 at the start and 1.21 from the first product on (the largest of a s + b s^3 + c s^5
// over [0, 1.21] is 1.2024), so elements of X and A = X X^T stay below 1.21 and 1.46,
// those of b A + c A^2 within 2.81.  e is chosen for these (kX, kA, kB); what lies
// below 2^-24 of the stored number's unit, 2^-38 of the largest, is lost.
//
// A row of a factor is a row of 128-byte lines, each the 32 high and then the 32
// low parts of 32 elements; rows are an odd number of lines apart, which spreads
// them over the L2.  Rows and columns are padded with zeros to multiples of 128.

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
#include "tiles.hpp"

using namespace mtdao;
using namespace mtdao::ops;

namespace {

constexpr int kThreads = 256;
constexpr int kChunk = 4096;   // elements that a workgroup sums the squares of at once
constexpr int kMostChunks = 1024;  // of a matrix, which every workgroup that splits it adds up
constexpr int kLine = 32;      // elements of a row in one line
constexpr int kPad = 128;      // rows and columns of a factor are multiples of this
constexpr int kMostParts = 12, kMostGemms = 2 * kMostParts;

// X <- a X + (b A + c A^2) X with A = X X^T.
constexpr double kCa = 3.4445, kCb = -4.7750, kCc = 2.0315;
// Exponents of the stored factors: X, A and A P, b A + c A^2, and Q - alpha I.
constexpr int kX = 14, kA = 14, kB = 13, kR = 10;
constexpr int kMostAtOnce = 3;  // steps that Q may stand for: kR suits Q up to a^3 = 40.9

typedef _Float16 v8h __attribute__((ext_vector_type(8)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// A matrix's row of the device table.
struct Row {
  void* p;
  const void* g;
  float* m;
  float decay, factor;
  int32_t rows, cols;
};

// Matrices of one shape: what the passes over elements need.
struct Part {
  uint8_t *natural, *turned;    // X and X^T of the first one: rows as the matrix's, and as its columns
  int64_t step;                 // bytes from one matrix's factors to the next one's
  int64_t rows, cols;           // of the matrix
  int32_t ld_natural, ld_turned;  // bytes
  int32_t matrix, count;        // the first one's place in the table, how many
  int32_t first_chunk, chunks;  // chunks of elements before these matrices, of each
  int32_t per_chunk;            // times kChunk elements
  int32_t first_tile, tiles_r, tiles_c;
};
struct Parts {
  Part part[kMostParts];
  int32_t n, items;
};

// Where the updates come from: rows of the table (Muon) or matrices one after another.
struct Source {
  const Row* rows;
  const void* x;
  double* sums;    // of every chunk
  float momentum;
  int32_t nesterov;
  double eps;
};

__device__ __forceinline__ int64_t item_of_launch() { return (int64_t)blockIdx.y * gridDim.x + blockIdx.x; }

// The update of N elements from the new momentum and the gradient.
template <int N>
__device__ __forceinline__ void update_of(const Source& s, const float (&g)[N], const float (&m)[N], float (&u)[N]) {
#pragma unroll
  for (int t = 0; t < N; ++t) u[t] = s.nesterov ? fmaf(s.momentum, m[t], g[t]) : m[t];
}

// Momentum (Muon) and the sum of the squares of a chunk of the update, in fp64.  Bound by HBM: 14 matrices
// of 2048 x 8192 with bf16 gradients 434 us, 5.4 TB/s.
constexpr int kSumV = 4;  // elements of a lane's vector: 16 bytes of momentum
template <typename GT, bool MUON>
__global__ __launch_bounds__(kThreads) void k_muon_sums(Parts parts, Source s) {
  __shared__ double part[kThreads / 64];
  const int64_t item = item_of_launch();
  if (item >= parts.items) return;
  int k = 0;
  while (k + 1 < parts.n && item >= parts.part[k + 1].first_chunk) ++k;
  const Part& a = parts.part[k];
  const int in = (int)(item - a.first_chunk), which = in / a.chunks;
  const int64_t numel = a.rows * a.cols, first = (int64_t)(in - which * a.chunks) * a.per_chunk * kChunk;
  const GT* g;
  float* m = nullptr;
  if (MUON) {
    g = reinterpret_cast<const GT*>(uniform_load(&s.rows[a.matrix + which].g));
    m = uniform_load(&s.rows[a.matrix + which].m);
  } else {
    g = reinterpret_cast<const GT*>(s.x) + (int64_t)(a.matrix + which) * numel;
  }
  constexpr int V = kSumV, kSlots = kChunk / (kThreads * V);
  double sum = 0.0;
  for (int64_t base = first; base < first + (int64_t)a.per_chunk * kChunk && base < numel; base += kChunk) {
    float ga[kSlots][V], ma[kSlots][V];
    int n[kSlots];
#pragma unroll
    for (int t = 0; t < kSlots; ++t) {
      const int64_t e = base + (t * kThreads + (int)threadIdx.x) * V, left = numel - e;
      n[t] = left > V ? V : (int)(left < 0 ? 0 : left);
      load_some<V>(g + e, n[t], ga[t]);
      if (MUON) load_some<V>(m + e, n[t], ma[t]);
    }
#pragma unroll
    for (int t = 0; t < kSlots; ++t) {
      float u[V];
      if (MUON) {
#pragma unroll
        for (int i = 0; i < V; ++i) ma[t][i] = fmaf(s.momentum, ma[t][i], ga[t][i]);
        if (n[t] > 0) store_some<V>(m + base + (t * kThreads + (int)threadIdx.x) * V, n[t], ma[t]);
        update_of(s, ga[t], ma[t], u);
      } else {
#pragma unroll
        for (int i = 0; i < V; ++i) u[i] = ga[t][i];
      }
#pragma unroll
      for (int i = 0; i < V; ++i) sum += (double)u[i] * (double)u[i];
    }
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o);
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = sum;
  __syncthreads();
  if (threadIdx.x == 0) s.sums[item] = (part[0] + part[1]) + (part[2] + part[3]);
}

// v as hi (low half of the word) and lo.
__device__ __forceinline__ uint32_t split_of(float v) {
  const _Float16 hi = (_Float16)v;
  const _Float16 lo = (_Float16)(v - (float)hi);
  return (uint32_t)__builtin_bit_cast(uint16_t, hi) | (uint32_t)__builtin_bit_cast(uint16_t, lo) << 16;
}
// Eight elements of a line, its chunk-th.
__device__ __forceinline__ void store_chunk(uint8_t* line, int chunk, const uint32_t (&w)[8]) {
  u32x4 hi, lo;
#pragma unroll
  for (int t = 0; t < 4; ++t) {
    hi[t] = __builtin_amdgcn_perm(w[2 * t + 1], w[2 * t], 0x05040100u);
    lo[t] = __builtin_amdgcn_perm(w[2 * t + 1], w[2 * t], 0x07060302u);
  }
  *reinterpret_cast<u32x4*>(line + chunk * 16) = hi;
  *reinterpret_cast<u32x4*>(line + 64 + chunk * 16) = lo;
}

// X and its transpose from the update: a tile of 64 x 64, whose transpose goes
// through LDS.  A thread has eight elements, a chunk of 16 bytes high and one low, of two rows, then of two columns.
// Every workgroup adds up the matrix's sums of squares, in an order that the sizes fix.
// Bound by HBM: the same 14 matrices 661 us, 5.0 TB/s (sixteen elements a thread, in pieces of 16 bytes
// 32 apart, 715 us).
constexpr int kSplit = 64;
template <typename GT, bool MUON>
__global__ __launch_bounds__(kThreads) void k_muon_split(Parts parts, Source s) {
  __shared__ uint32_t tile[kSplit][kSplit + 1];
  __shared__ double part[kThreads / 64];
  const int64_t item = item_of_launch();
  if (item >= parts.items) return;
  int k = 0;
  while (k + 1 < parts.n && item >= parts.part[k + 1].first_tile) ++k;
  const Part& a = parts.part[k];
  const int in = (int)(item - a.first_tile), tiles = a.tiles_r * a.tiles_c, which = in / tiles, at = in - which * tiles;
  const int64_t row0 = (int64_t)(at / a.tiles_c) * kSplit, col0 = (int64_t)(at % a.tiles_c) * kSplit;
  const int line = threadIdx.x / 8, chunk = threadIdx.x % 8;
  const GT* g;
  const float* m = nullptr;
  if (MUON) {
    g = reinterpret_cast<const GT*>(uniform_load(&s.rows[a.matrix + which].g));
    m = uniform_load(&s.rows[a.matrix + which].m);
  } else {
    g = reinterpret_cast<const GT*>(s.x) + (int64_t)(a.matrix + which) * a.rows * a.cols;
  }
  float u[2][8];
  int n[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int64_t row = row0 + h * 32 + line, col = col0 + chunk * 8, e = row * a.cols + col, left = row < a.rows ? a.cols - col : 0;
    n[h] = left < 0 ? 0 : left > 8 ? 8 : (int)left;
    load_some<8>(g + e, n[h], u[h]);
    if (MUON) {
      float ma[8];
      load_some<8>(m + e, n[h], ma);
      update_of(s, u[h], ma, u[h]);
    }
  }
  const double* from = s.sums + a.first_chunk + (int64_t)which * a.chunks;
  double sum = 0.0;
#pragma unroll 4
  for (int i = threadIdx.x; i < a.chunks; i += kThreads) sum += from[i];
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o);
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = sum;
  __syncthreads();
  const double scale = (double)(1 << kX) / (sqrt((part[0] + part[1]) + (part[2] + part[3])) + s.eps);
  const int64_t own = (int64_t)which * a.step;
  uint32_t w[8];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
#pragma unroll
    for (int t = 0; t < 8; ++t) {
      w[t] = t < n[h] ? split_of((float)((double)u[h][t] * scale)) : 0u;
      tile[h * 32 + line][chunk * 8 + t] = w[t];
    }
    store_chunk(a.natural + own + (row0 + h * 32 + line) * a.ld_natural + (col0 + chunk * 8) / kLine * 128, chunk % 4, w);
  }
  __syncthreads();
#pragma unroll
  for (int h = 0; h < 2; ++h) {
#pragma unroll
    for (int t = 0; t < 8; ++t) w[t] = tile[chunk * 8 + t][h * 32 + line];
    store_chunk(a.turned + own + (col0 + h * 32 + line) * a.ld_turned + (row0 + chunk * 8) / kLine * 128, chunk % 4, w);
  }
}

// ------------------------------------------------------------------ products

// c = k0 a b^T + k1 d1 + k2 d2 of `count` matrices: as a factor (out, and its transpose in
// turned), or as the result of the last product.
struct Gemm {
  const uint8_t *a, *b, *d1, *d2;
  uint8_t *out, *turned;
  int64_t step;               // bytes from one matrix's factors to the next one's
  int64_t rows, cols;         // of the result, without padding (last product)
  int32_t rows_a, rows_b, blocks;  // padded rows, lines of the contraction
  int32_t lda, ldb, ldo, ldt;      // bytes; d1 and d2 have out's rows
  int32_t symmetric;          // tiles on and above the diagonal only, out is turned
  int32_t tiles_a, tiles_b, tiles;
  int32_t parts, part_blocks; // of the contraction, and their lines
  float* partial;             // with more than one part: their sums, a tile after another, its parts together
  int32_t count, matrix;      // matrices, the first one's place in the table
  int32_t first, share;       // an XCD's tiles before its share of these matrices' tiles, that share
  int32_t last;
  float k0, k1, k2;
};
struct Gemms {
  Gemm gemm[kMostGemms];
  int32_t n;
};
struct Last {
  const Row* rows;   // Muon's table
  void* out;         // or matrices one after another
  float lr;
};

// Fragments of 32 x 32 go between lanes, each with sixteen elements of a row, and memory, in whole lines, by way of
// LDS of the wave's own: 32 lines, then 32 rows of 33 words to turn a fragment.  (Pieces of 16 bytes straight from the
// lanes take four times as many cycles of the CU's path to memory.)
constexpr int kStaged = 32 * 128, kOwn = kStaged + 32 * 33 * 4;
__device__ __forceinline__ u32x4* staged_at(uint8_t* mine, int row, int chunk) {
  return reinterpret_cast<u32x4*>(mine + row * 128 + ((chunk ^ row_key(row)) << 4));
}
__device__ __forceinline__ void load_lines(const uint8_t* from, int ld, int lane, u32x4 (&w)[4]) {
#pragma unroll
  for (int k = 0; k < 4; ++k) w[k] = *reinterpret_cast<const u32x4*>(from + (int64_t)(k * 8 + lane / 8) * ld + lane % 8 * 16);
}
__device__ __forceinline__ void staged_in(uint8_t* mine, int lane, const u32x4 (&w)[4], float (&v)[16]) {
  const int fr = lane % 32, fg = lane / 32;
  lanes_done();
#pragma unroll
  for (int k = 0; k < 4; ++k) *staged_at(mine, k * 8 + lane / 8, lane % 8) = w[k];
  lanes_done();
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const v8h hi = __builtin_bit_cast(v8h, *staged_at(mine, fr, 2 * fg + h)), lo = __builtin_bit_cast(v8h, *staged_at(mine, fr, 4 + 2 * fg + h));
#pragma unroll
    for (int t = 0; t < 8; ++t) v[8 * h + t] = (float)hi[t] + (float)lo[t];
  }
}
__device__ __forceinline__ void staged_out(uint8_t* mine, int lane, const uint32_t (&w)[16], uint8_t* to, int ld) {
  const int fr = lane % 32, fg = lane / 32;
  lanes_done();
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    u32x4 hi, lo;
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      hi[t] = __builtin_amdgcn_perm(w[8 * h + 2 * t + 1], w[8 * h + 2 * t], 0x05040100u);
      lo[t] = __builtin_amdgcn_perm(w[8 * h + 2 * t + 1], w[8 * h + 2 * t], 0x07060302u);
    }
    *staged_at(mine, fr, 2 * fg + h) = hi;
    *staged_at(mine, fr, 4 + 2 * fg + h) = lo;
  }
  lanes_done();
#pragma unroll
  for (int k = 0; k < 4; ++k) *reinterpret_cast<u32x4*>(to + (int64_t)(k * 8 + lane / 8) * ld + lane % 8 * 16) = *staged_at(mine, k * 8 + lane / 8, lane % 8);
}
__device__ __forceinline__ void turn_fragment(uint32_t* words, int lane, uint32_t (&w)[16]) {
  const int fr = lane % 32, fg = lane / 32;
  lanes_done();
#pragma unroll
  for (int t = 0; t < 16; ++t) words[fr * 33 + fg * 16 + t] = w[t];
  lanes_done();
#pragma unroll
  for (int t = 0; t < 16; ++t) w[t] = words[(fg * 16 + t) * 33 + fr];
}

// Tile (i, j) of the tiles on and above the diagonal of n x n, row by row.
__device__ __forceinline__ void triangle_place(int t, int n, int& i, int& j) {
  i = 0;
  while (t >= n - i) t -= n - i++;
  j = i + t;
}

// A fragment of the last result, by way of LDS as above: four consecutive elements of a row a lane,
// in four rows.
struct Spot {
  int64_t at;   // of the first row's four elements
  int n, rows;  // of these that there are; rows from the first one on
};
__device__ __forceinline__ Spot spot_of(const Gemm& q, int lane, int r0, int c0) {
  const int64_t row = r0 + lane / 8, col = c0 + lane % 8 * 4, left = q.cols - col, rows = q.rows - row;
  return {row * q.cols + col, left > 4 ? 4 : left < 0 ? 0 : (int)left, rows > 32 ? 32 : rows < 0 ? 0 : (int)rows};
}
template <typename PT>
__device__ __forceinline__ void load_last(const Gemm& q, const PT* p, const Spot& spot, float (&v)[4][4]) {
#pragma unroll
  for (int k = 0; k < 4; ++k) load_some<4>(p + spot.at + k * 8 * q.cols, k * 8 < spot.rows ? spot.n : 0, v[k]);
}
// keep p + step v; keep and step are not looked at without `onto`: then v
template <typename PT>
__device__ __forceinline__ void store_last(const Gemm& q, PT* p, const Spot& spot, uint8_t* mine, int lane, const float (&v)[16], const float (&before)[4][4], bool onto,
                                           float keep, float step) {
  const int fr = lane % 32, fg = lane / 32;
  lanes_done();
#pragma unroll
  for (int k = 0; k < 4; ++k) *staged_at(mine, fr, 4 * fg + k) = __builtin_bit_cast(u32x4, v4f{v[4 * k], v[4 * k + 1], v[4 * k + 2], v[4 * k + 3]});
  lanes_done();
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const v4f made = __builtin_bit_cast(v4f, *staged_at(mine, k * 8 + lane / 8, lane % 8));
    float o[4];
#pragma unroll
    for (int t = 0; t < 4; ++t) o[t] = onto ? fmaf(step, made[t], before[k][t] * keep) : made[t];
    if (k * 8 < spot.rows && spot.n > 0) store_some<4>(p + spot.at + k * 8 * q.cols, spot.n, o);
  }
}

// The products of a launch in tiles of B x B over WR x WC waves, a tile a workgroup.
// Rows of b go in as the instruction's rows, so that a lane ends with sixteen
// consecutive columns of a row of c.
//
// LDS holds STAGES lines of each row of both sides, loaded straight into it.  A line is
// two steps of sixteen elements; a wave reads a step's fragments while the matrix
// cores work on the step before, so it needs others only once a line: before the last step, when the line's last
// fragments are in registers, all meet; then its place is free to be loaded, and the next line is there.
//
// Bound, with tiles of 256, by the matrix cores and the power they draw: A = X X^T of 14 matrices of 2048 x 8192
// 1.2 ms, 1.35 PFLOP/s of the three instructions (a library's plain fp16 product of 8192^3: 1.06); squares 355 us, 1.14, and
// products with X 2.6 ms, 1.11, as what a tile adds to and writes, 512 KB in some 30 us, goes by with
// nothing behind it (one workgroup a CU).  Small products are bound by latency: 5 us a launch of one tile a CU, and
// 0.2 us a line.
template <int B, int WR, int WC, int STAGES, typename PT>
__global__ __launch_bounds__(64 * WR * WC, 2) void k_muon_product(Gemms all, Last last) {
  constexpr int kWaves = WR * WC, kMI = B / WR / 32, kNI = B / WC / 32, kLoads = B / (8 * kWaves), kStage = 2 * B * 128;
  constexpr int kFragments = 2 * (kMI + kNI), kCalls = 3 * kMI * kNI, kSums = kMI * kNI == 1 ? 3 : 1;
  static_assert((STAGES & (STAGES - 1)) == 0 && STAGES >= 2 && STAGES * 2 * kLoads <= 63, "stages are told by bits, loads in flight counted");
  extern __shared__ __attribute__((aligned(1024))) uint8_t lds[];
  const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  // Workgroups go to the eight XCDs in turn.  Each takes its eighth of the tiles of every
  // shape, so that all have as much to do, in neighbouring tiles, which share rows in its L2.
  const int turn = (int)(blockIdx.x / 8);
  int k = 0;
  while (k + 1 < all.n && turn >= all.gemm[k + 1].first) ++k;
  const Gemm& q = all.gemm[k];
  const int in = (int)(blockIdx.x % 8) * q.share + turn - q.first, of_all = in / q.parts, part = in - of_all * q.parts;
  const int which = of_all / q.tiles, tile = of_all - which * q.tiles;
  if (which >= q.count) return;
  int ti, tj;
  if (q.symmetric) {
    triangle_place(tile, q.tiles_a, ti, tj);
  } else {
    ti = tile % q.tiles_a;
    tj = tile / q.tiles_a;
  }
  const int row0 = ti * B, col0 = tj * B, from = part * q.part_blocks;
  const int blocks = q.blocks - from < q.part_blocks ? q.blocks - from : q.part_blocks;
  const int64_t own = (int64_t)which * q.step;

  // A wave loads eight rows at once: lane l the chunk that belongs at place l % 8 of row l / 8.
  const int lr = wave * 8 + lane / 8, lda = q.lda, ldb = q.ldb;
  const auto ra = buffer_of(q.a + own + (int64_t)row0 * lda, (int64_t)(q.rows_a - row0) * lda);
  const auto rb = buffer_of(q.b + own + (int64_t)col0 * ldb, (int64_t)(q.rows_b - col0) * ldb);
  int va = lr * lda + ((lane % 8) ^ row_key(lr)) * 16, vb = lr * ldb + ((lane % 8) ^ row_key(lr)) * 16;
  auto load_part = [&](int t, int block) {  // 0 .. 2 kLoads - 1: those of a, then those of b
    const bool of_b = t >= kLoads;
    const int line = from + (block < blocks ? block : blocks - 1);  // (past the last line it is loaded again, and not used)
    asm("" : "+v"(va), "+v"(vb));  // (offsets of further rows are formed anew: they would each hold a register)
    __builtin_amdgcn_raw_ptr_buffer_load_lds(
        of_b ? rb : ra, (__attribute__((address_space(3))) void*)(lds + (block & (STAGES - 1)) * kStage + wave * 1024 + t * kWaves * 1024), 16,
        of_b ? vb + (t - kLoads) * 8 * kWaves * ldb : va + t * 8 * kWaves * lda, line * 128, 0, 0);
  };

  const int wm = wave / WC * (32 * kMI), wn = wave % WC * (32 * kNI), fr = lane % 32, fg = lane / 32;
  const int key_a = row_key(wm + fr), key_b = row_key(wn + row_of_b(fr));
  const int a0 = (wm + fr) * 128 + ((fg ^ key_a) << 4), b0 = (B + wn + row_of_b(fr)) * 128 + ((fg ^ key_b) << 4);
  // Fragments of a step: of b high, of a high, of b low, of a low, in the order of their use.
  v8h f[2][kFragments];
  auto read_part = [&](int t, int stage, int step, int to) {
    const bool low = t >= kMI + kNI;
    const int r = low ? t - kMI - kNI : t, chunk = (low ? 64 : 0) ^ step * 32;
    f[to][t] = *reinterpret_cast<const v8h*>(lds + stage * kStage + (r < kNI ? (b0 ^ chunk) + r * 4096 : (a0 ^ chunk) + (r - kNI) * 4096));
  };
  v16f acc[kSums][kMI][kNI];
#pragma unroll
  for (int k = 0; k < kSums; ++k)
#pragma unroll
    for (int i = 0; i < kMI; ++i)
#pragma unroll
      for (int j = 0; j < kNI; ++j)
#pragma unroll
        for (int t = 0; t < 16; ++t) acc[k][i][j][t] = 0.0f;
#pragma unroll
  for (int s = 0; s < STAGES; ++s)
#pragma unroll
    for (int t = 0; t < 2 * kLoads; ++t) load_part(t, s);
  loads_landed<(STAGES - 1) * 2 * kLoads>();
  meet();
#pragma unroll
  for (int t = 0; t < kFragments; ++t) read_part(t, 0, 0, 0);
  for (int block = 0; block < blocks; ++block) {
    const int stage = block & (STAGES - 1), after = (block + 1) & (STAGES - 1);
#pragma unroll
    for (int step = 0; step < 2; ++step) {
      if (step == 1) {
        reads_landed();
        loads_landed<(STAGES - 2) * 2 * kLoads>();
        meet();
      }
#pragma unroll
      for (int c = 0; c < kCalls; ++c) {
        // high high, low high, high low: the same sums come up again after kMI kNI instructions (a single one has one for each)
        const int kind = c / (kMI * kNI), i = c % (kMI * kNI) / kNI, j = c % kNI;
        const v8h& fb = f[step][(kind == 1 ? kMI + kNI : 0) + j];
        const v8h& fa = f[step][(kind == 2 ? kMI + kNI : 0) + kNI + i];
        v16f& sum = acc[kSums == 3 ? kind : 0][i][j];
        sum = __builtin_amdgcn_mfma_f32_32x32x16_f16(fb, fa, sum, 0, 0, 0);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int t = 0; t < kFragments; ++t)
          if (t * kCalls / kFragments == c) read_part(t, step == 0 ? stage : after, step ^ 1, step ^ 1);
        if (step == 1) {
#pragma unroll
          for (int t = 0; t < 2 * kLoads; ++t)
            if (t * kCalls / (2 * kLoads) == c) load_part(t, block + STAGES);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
#pragma unroll
      for (int k = 0; k < kSums; ++k)
#pragma unroll
        for (int i = 0; i < kMI; ++i)
#pragma unroll
          for (int j = 0; j < kNI; ++j) asm volatile("" : "+v"(acc[k][i][j]));  // (without a use here the instructions would be moved past the next barrier)
    }
  }
  // (past the last line its fragments are read again, and not used)
  reads_landed();
  loads_landed();
  meet();
  if constexpr (kSums == 3) {
    if (q.parts > 1) {
      float* to = q.partial + (int64_t)in * (B * B) + wave * 1024 + lane;
#pragma unroll
      for (int t = 0; t < 16; ++t) to[t * 64] = acc[0][0][0][t] + (acc[1][0][0][t] + acc[2][0][0][t]);
      return;
    }
  }
  uint8_t* mine = lds + wave * kOwn;
  uint8_t* turned = q.symmetric ? (ti == tj ? nullptr : q.out) : q.turned;
  const int ldt = q.symmetric ? q.ldo : q.ldt;
  auto place = [&](int f, int& r0, int& c0) {
    r0 = row0 + wm + f / kNI * 32;
    c0 = col0 + wn + f % kNI * 32;
    return r0 < q.rows_a && c0 < q.rows_b;
  };
  // (what the next fragment adds to is on its way while one is worked on)
  u32x4 ahead[4];
  float before[4][4];
  const bool onto = last.rows != nullptr;
  PT* p = nullptr;
  float keep = 0.0f, step = 0.0f;
  if (q.last) {
    if (onto) {
      const Row& r = last.rows[q.matrix + which];
      p = reinterpret_cast<PT*>(r.p);
      keep = 1.0f - last.lr * r.decay;
      step = -last.lr * r.factor;
    } else {
      p = reinterpret_cast<PT*>(last.out) + (int64_t)(q.matrix + which) * q.rows * q.cols;
    }
  }
  auto fetch = [&](int f) {
    int r0, c0;
    if (!place(f, r0, c0)) return;
    if (q.d1) load_lines(q.d1 + own + (int64_t)r0 * q.ldo + c0 / kLine * 128, q.ldo, lane, ahead);
  };
  auto fetch_last = [&](int f) {
    int r0, c0;
    if (q.last && onto && place(f, r0, c0)) load_last(q, p, spot_of(q, lane, r0, c0), before);
  };
  fetch(0);
  fetch_last(0);
#pragma unroll
  for (int f = 0; f < kMI * kNI; ++f) {
    const int i = f / kNI, j = f % kNI;
    int r0, c0;
    if (!place(f, r0, c0)) continue;
    const int64_t line = own + (int64_t)r0 * q.ldo + c0 / kLine * 128;
    float v[16], d[16];
#pragma unroll
    for (int t = 0; t < 16; ++t) v[t] = q.k0 * (kSums == 3 ? acc[0][i][j][t] + (acc[kSums / 2][i][j][t] + acc[kSums - 1][i][j][t]) : acc[0][i][j][t]);
    if (q.d1) {
      staged_in(mine, lane, ahead, d);
      if (f + 1 < kMI * kNI) fetch(f + 1);
#pragma unroll
      for (int t = 0; t < 16; ++t) v[t] = fmaf(q.k1, d[t], v[t]);
    }
    if (q.d2) {
      u32x4 now[4];
      load_lines(q.d2 + line, q.ldo, lane, now);
      staged_in(mine, lane, now, d);
#pragma unroll
      for (int t = 0; t < 16; ++t) v[t] = fmaf(q.k2, d[t], v[t]);
    }
    if (q.last) {
      float now[4][4];
#pragma unroll
      for (int k = 0; k < 4; ++k)
#pragma unroll
        for (int t = 0; t < 4; ++t) now[k][t] = before[k][t];
      if (f + 1 < kMI * kNI) fetch_last(f + 1);
      store_last(q, p, spot_of(q, lane, r0, c0), mine, lane, v, now, onto, keep, step);
      continue;
    }
    uint32_t w[16];
#pragma unroll
    for (int t = 0; t < 16; ++t) w[t] = split_of(v[t]);
    staged_out(mine, lane, w, q.out + line, q.ldo);
    if (turned) {
      turn_fragment(reinterpret_cast<uint32_t*>(mine + kStaged), lane, w);
      staged_out(mine, lane, w, turned + own + (int64_t)c0 * ldt + r0 / kLine * 128, ldt);
    }
  }
}

// A = X X^T from the sums of its parts, added in their order: a tile of 64 x 64 a workgroup.
__global__ __launch_bounds__(256) void k_muon_join(Gemms all) {
  constexpr int B = 64;
  __shared__ __attribute__((aligned(128))) uint8_t lds[4 * kOwn];
  const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  int in = blockIdx.x, k = 0;
  for (; k < all.n; ++k) {
    const int here = all.gemm[k].parts > 1 ? all.gemm[k].tiles * all.gemm[k].count : 0;
    if (in < here) break;
    in -= here;
  }
  if (k == all.n) return;
  const Gemm& q = all.gemm[k];
  const int which = in / q.tiles;
  int ti, tj;
  triangle_place(in - which * q.tiles, q.tiles_a, ti, tj);
  const float* from = q.partial + (int64_t)in * q.parts * (B * B) + wave * 1024 + lane;
  float v[16] = {};
#pragma unroll 4
  for (int part = 0; part < q.parts; ++part) {
#pragma unroll
    for (int t = 0; t < 16; ++t) v[t] += from[part * (B * B) + t * 64];
  }
  uint32_t w[16];
#pragma unroll
  for (int t = 0; t < 16; ++t) w[t] = split_of(q.k0 * v[t]);
  uint8_t *mine = lds + wave * kOwn, *out = q.out + (int64_t)which * q.step;
  const int r0 = ti * B + wave / 2 * 32, c0 = tj * B + wave % 2 * 32;
  staged_out(mine, lane, w, out + (int64_t)r0 * q.ldo + c0 / kLine * 128, q.ldo);
  if (ti == tj) return;
  turn_fragment(reinterpret_cast<uint32_t*>(mine + kStaged), lane, w);
  staged_out(mine, lane, w, out + (int64_t)c0 * q.ldo + r0 / kLine * 128, q.ldo);
}

// ------------------------------------------------------------ small matrices

// Matrices of up to 64 x 256 (or 256 x 64), all of whose work one workgroup does: X and its transpose
// lie in LDS, lines as in memory, A and then b A + c A A in a third place; X, to which each step adds,
// also in registers, as the fp32 it is formed in.  Wave w has the w-th 32 columns of X, the first one
// to three waves the blocks of A on and above the diagonal.  MB: blocks of X's rows.
// Bound by latency, of the steps' four or five meetings, chains of matrix instructions and what is written both ways: 64 x 64
// 24 us, 64 x 256 38 us; 100 x 37 25 us.  (Replayed, so / through the launches that large matrices take: 64 x 64 28 / 85 us,
// 64 x 256 44 / 89, 200 of them 50 / 241, 1000 182 / 1149.)
constexpr int kTinyM = 64, kTinyN = 256, kTinyThreads = 512;

// Parts of X's lines in which A = X X^T is formed: eight waves among its one or three blocks.
template <int MB>
constexpr int kTinyParts = MB == 1 ? 8 : 2;

struct Tiny {
  int32_t first, lines;   // of the table; lines of X's rows
  int64_t rows, cols;     // matrices one after another (no table)
  int32_t steps;
};

// Chunk `chunk` (16 bytes) of line `line` in a row of LINES lines.  Rows lie 256 bytes, all banks, or a multiple
// apart where there are more than one: then the row's last bit swaps neighbouring lines.
template <bool ONE>
__device__ __forceinline__ int chunk_at(int row, int line, int chunk, int stride) {
  return row * stride + (ONE ? line : line ^ (row & 1)) * 128 + ((chunk ^ row_key(row)) << 4);
}

template <typename GT, typename PT, bool MUON, int MB>
__global__ __launch_bounds__(kTinyThreads) void k_muon_tiny(Tiny t, Source s, Last last) {
  extern __shared__ __attribute__((aligned(1024))) uint8_t lds[];
  __shared__ double part[kTinyThreads / 64];
  constexpr int kM = 32 * MB, kBlocks = MB * (MB + 1) / 2, kParts = kTinyParts<MB>;
  const int tid = (int)threadIdx.x, lane = tid % 64, wave = __builtin_amdgcn_readfirstlane(tid / 64), fr = lane % 32, fg = lane / 32;
  const int xs = t.lines * 128, ts = MB * 128;      // bytes of a row of X, and of X^T and A
  uint8_t *X = lds, *T = X + kM * xs, *A = T + t.lines * kLine * ts;
  float* sums = reinterpret_cast<float*>(A + kM * ts);  // of A's parts but the first
  const int which = t.first + (int)blockIdx.x;
  const Row* entry = MUON ? s.rows + which : nullptr;
  const int r = MUON ? entry->rows : (int)t.rows, c = MUON ? entry->cols : (int)t.cols;
  const bool tall = r > c;
  const int n = tall ? r : c, blocks = (n + kLine - 1) / kLine;  // columns of X
  const GT* g;
  float* mom = nullptr;
  if (MUON) {
    g = reinterpret_cast<const GT*>(entry->g);
    mom = entry->m;
  } else {
    g = reinterpret_cast<const GT*>(s.x) + (int64_t)which * r * c;
  }
  auto at_x = [&](int row, int line, int chunk) { return X + chunk_at<false>(row, line, chunk, xs); };
  auto at_t = [&](int row, int line, int chunk) { return T + chunk_at<MB == 1>(row, line, chunk, ts); };
  auto at_a = [&](int row, int line, int chunk) { return A + chunk_at<MB == 1>(row, line, chunk, ts); };
  // one element of a row, hi and lo
  auto put = [&](auto at, int row, int col, uint32_t w) {
    *reinterpret_cast<uint16_t*>(at(row, col / kLine, col % kLine / 8) + col % 8 * 2) = (uint16_t)w;
    *reinterpret_cast<uint16_t*>(at(row, col / kLine, 4 + col % kLine / 8) + col % 8 * 2) = (uint16_t)(w >> 16);
  };

  for (int i = tid; i < (kM * xs + t.lines * kLine * ts) / 16; i += kTinyThreads) reinterpret_cast<u32x4*>(lds)[i] = u32x4{0, 0, 0, 0};
  constexpr int kSlots = kTinyM * kTinyN / 8 / kTinyThreads;
  const int vectors = (c + 7) / 8, all = r * vectors;
  float u[kSlots][8];
  double sum = 0.0;
#pragma unroll
  for (int q = 0; q < kSlots; ++q) {
    const int v = q * kTinyThreads + tid, row = v / vectors, col = (v - row * vectors) * 8, e = row * c + col;
    const int live = v < all ? (c - col > 8 ? 8 : c - col) : 0;
    load_some<8>(g + e, live, u[q]);
    if (MUON) {
      float m[8];
      load_some<8>(mom + e, live, m);
#pragma unroll
      for (int i = 0; i < 8; ++i) m[i] = fmaf(s.momentum, m[i], u[q][i]);
      if (live > 0) store_some<8>(mom + e, live, m);
      update_of(s, u[q], m, u[q]);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) sum += (double)u[q][i] * (double)u[q][i];
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o);
  if (lane == 0) part[wave] = sum;
  __syncthreads();
  sum = 0.0;
#pragma unroll
  for (int w = 0; w < kTinyThreads / 64; ++w) sum += part[w];
  const double scale = (double)(1 << kX) / (sqrt(sum) + s.eps);
#pragma unroll
  for (int q = 0; q < kSlots; ++q) {
    const int v = q * kTinyThreads + tid, row = v / vectors, col = (v - row * vectors) * 8;
    if (v >= all) continue;
    uint32_t w[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = split_of((float)((double)u[q][i] * scale));  // (zeros past the row's end)
    // a chunk in the row's place, an element in each of eight rows of the transpose
    auto both = [&](auto at_own, auto at_turned) {
      u32x4 hi, lo;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        hi[i] = __builtin_amdgcn_perm(w[2 * i + 1], w[2 * i], 0x05040100u);
        lo[i] = __builtin_amdgcn_perm(w[2 * i + 1], w[2 * i], 0x07060302u);
      }
      *reinterpret_cast<u32x4*>(at_own(row, col / kLine, col % kLine / 8)) = hi;
      *reinterpret_cast<u32x4*>(at_own(row, col / kLine, 4 + col % kLine / 8)) = lo;
#pragma unroll
      for (int i = 0; i < 8; ++i) put(at_turned, col + i, row, w[i]);  // (rows there are for whole chunks)
    };
    if (tall) both(at_t, at_x);
    else both(at_x, at_t);
  }
  __syncthreads();

  // sums of hi hi, lo hi and hi lo of 32 rows of a and of b over lines from .. to; a line's eight
  // fragments are read while the one before is multiplied
  auto product = [&](auto at_rows, int row0, auto at_cols, int col0, int from, int to, float (&v)[16]) {
    v16f acc[3];
#pragma unroll
    for (int k = 0; k < 3; ++k)
#pragma unroll
      for (int i = 0; i < 16; ++i) acc[k][i] = 0.0f;
    const int ra = row0 + fr, rb = col0 + row_of_b(fr);
    v8h now[2][4], next[2][4];
    auto read = [&](int line, v8h (&f)[2][4]) {
#pragma unroll
      for (int step = 0; step < 2; ++step)
#pragma unroll
        for (int low = 0; low < 2; ++low) {
          f[step][low] = *reinterpret_cast<const v8h*>(at_rows(ra, line, 4 * low + 2 * step + fg));
          f[step][2 + low] = *reinterpret_cast<const v8h*>(at_cols(rb, line, 4 * low + 2 * step + fg));
        }
    };
    if (from < to) read(from, now);
    for (int line = from; line < to; ++line) {
      if (line + 1 < to) read(line + 1, next);
#pragma unroll
      for (int step = 0; step < 2; ++step) {
        acc[0] = __builtin_amdgcn_mfma_f32_32x32x16_f16(now[step][2], now[step][0], acc[0], 0, 0, 0);
        acc[1] = __builtin_amdgcn_mfma_f32_32x32x16_f16(now[step][3], now[step][0], acc[1], 0, 0, 0);
        acc[2] = __builtin_amdgcn_mfma_f32_32x32x16_f16(now[step][2], now[step][1], acc[2], 0, 0, 0);
      }
#pragma unroll
      for (int step = 0; step < 2; ++step)
#pragma unroll
        for (int k = 0; k < 4; ++k) now[step][k] = next[step][k];
    }
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = acc[0][i] + (acc[1][i] + acc[2][i]);
  };
  // a block's values as a factor (row fr, sixteen columns), and, turned, in another place
  auto store_block = [&](auto at, int row0, int col0, const uint32_t (&w)[16]) {
    u32x4 hi[2], lo[2];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      hi[i / 4][i % 4] = __builtin_amdgcn_perm(w[2 * i + 1], w[2 * i], 0x05040100u);
      lo[i / 4][i % 4] = __builtin_amdgcn_perm(w[2 * i + 1], w[2 * i], 0x07060302u);
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      *reinterpret_cast<u32x4*>(at(row0 + fr, col0 / kLine, 2 * fg + h)) = hi[h];
      *reinterpret_cast<u32x4*>(at(row0 + fr, col0 / kLine, 4 + 2 * fg + h)) = lo[h];
    }
  };
  // (two lanes share what they hold of two rows, so that each stores pairs in one of them: halves of words cost
  // LDS as much as words, and twice where both halves come at once)
  auto store_turned = [&](auto at, int row0, int col0, const uint32_t (&w)[16]) {
    const bool odd = fr & 1;
    const int col = row0 + (fr & ~1);
#pragma unroll
    for (int i = 0; i < 16; i += 2) {
      const uint32_t own = odd ? w[i + 1] : w[i];
      const uint32_t other = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(odd ? w[i] : w[i + 1]), 0xb1, 0xf, 0xf, true);  // of the neighbour
      const uint32_t first = odd ? other : own, second = odd ? own : other;
      const int row = col0 + fg * 16 + i + odd;
      *reinterpret_cast<uint32_t*>(at(row, col / kLine, col % kLine / 8) + col % 8 * 2) = __builtin_amdgcn_perm(second, first, 0x05040100u);
      *reinterpret_cast<uint32_t*>(at(row, col / kLine, 4 + col % kLine / 8) + col % 8 * 2) = __builtin_amdgcn_perm(second, first, 0x07060302u);
    }
  };
  // the block of A of a wave, and its part of X's lines where there are many
  const int block = wave % kBlocks, mine = wave / kBlocks, parts = blocks > 2 ? kParts : 1, part_lines = (blocks + parts - 1) / parts;
  const int bi = block == 2 ? 32 : 0, bj = MB == 1 || block == 0 ? 0 : 32;
  auto store_square = [&](const float (&v)[16]) {
    uint32_t w[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) w[i] = split_of(v[i]);
    store_block(at_a, bi, bj, w);
    if (bi != bj) store_turned(at_a, bi, bj, w);
  };

  float x[MB][16];
  if (wave < blocks) {
#pragma unroll
    for (int b = 0; b < MB; ++b)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const v8h hi = *reinterpret_cast<const v8h*>(at_x(32 * b + fr, wave, 2 * fg + h)), lo = *reinterpret_cast<const v8h*>(at_x(32 * b + fr, wave, 4 + 2 * fg + h));
#pragma unroll
        for (int i = 0; i < 8; ++i) x[b][8 * h + i] = (float)hi[i] + (float)lo[i];
      }
  }
  for (int step = 0; step < t.steps; ++step) {
    float gram[16], poly[16];
    if (mine < parts) {
      const int from = mine * part_lines, to = from + part_lines < blocks ? from + part_lines : blocks;
      product(at_x, bi, at_x, bj, from, to, gram);
      if (mine > 0) {
#pragma unroll
        for (int i = 0; i < 16; ++i) sums[((mine - 1) * kBlocks + block) * 1024 + i * 64 + lane] = gram[i];
      }
    }
    if (parts > 1) __syncthreads();
    if (wave < kBlocks) {
      for (int part = 1; part < parts; ++part)
#pragma unroll
        for (int i = 0; i < 16; ++i) gram[i] += sums[((part - 1) * kBlocks + block) * 1024 + i * 64 + lane];
#pragma unroll
      for (int i = 0; i < 16; ++i) gram[i] *= __builtin_ldexpf(1.0f, kA - 2 * kX);
      store_square(gram);
    }
    __syncthreads();
    if (wave < kBlocks) {
      product(at_a, bi, at_a, bj, 0, MB, poly);
#pragma unroll
      for (int i = 0; i < 16; ++i)
        poly[i] = fmaf((float)kCb * __builtin_ldexpf(1.0f, kB - kA), gram[i], (float)kCc * __builtin_ldexpf(1.0f, kB - 2 * kA) * poly[i]);
    }
    __syncthreads();
    if (wave < kBlocks) store_square(poly);
    __syncthreads();
    if (wave < blocks) {
#pragma unroll
      for (int b = 0; b < MB; ++b) {
        float v[16];
        product(at_a, 32 * b, at_t, 32 * wave, 0, MB, v);
#pragma unroll
        for (int i = 0; i < 16; ++i) x[b][i] = fmaf((float)kCa, x[b][i], __builtin_ldexpf(1.0f, -kB) * v[i]);
      }
      if (step + 1 < t.steps) {  // (X^T is read by this wave alone, and all of X's blocks are formed)
#pragma unroll
        for (int b = 0; b < MB; ++b) {
          uint32_t w[16];
#pragma unroll
          for (int i = 0; i < 16; ++i) w[i] = split_of(x[b][i]);
          store_block(at_x, 32 * b, 32 * wave, w);
          store_turned(at_t, 32 * b, 32 * wave, w);
        }
      }
    }
    __syncthreads();
  }
  if (wave >= blocks) return;
  PT* out = MUON ? reinterpret_cast<PT*>(entry->p) : reinterpret_cast<PT*>(last.out) + (int64_t)which * r * c;
  const float keep = MUON ? 1.0f - last.lr * entry->decay : 0.0f, move = MUON ? -last.lr * entry->factor : 0.0f;
#pragma unroll
  for (int b = 0; b < MB; ++b) {
    if (tall) {  // a column's sixteen rows a lane, neighbouring columns in neighbouring lanes
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int row = 32 * wave + fg * 16 + i, col = 32 * b + fr;
        if (row < r && col < c) {
          PT* at = out + row * c + col;
          const float o = __builtin_ldexpf(1.0f, -kX) * x[b][i];
          store_one(at, MUON ? fmaf(move, o, to_f32(*at) * keep) : o);
        }
      }
    } else {
      const int row = 32 * b + fr;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int col = 32 * wave + fg * 16 + 8 * h, n = row < r ? c - col : 0;
        if (n <= 0) continue;
        PT* at = out + row * c + col;
        float o[8];
        if (MUON) load_some<8>(at, n, o);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float made = __builtin_ldexpf(1.0f, -kX) * x[b][8 * h + i];
          o[i] = MUON ? fmaf(move, made, o[i] * keep) : made;
        }
        store_some<8>(at, n, o);
      }
    }
  }
}

// Writes rows `at`.. of the table.
constexpr int kRowsAtOnce = 64;
struct Rows {
  Row row[kRowsAtOnce];
};
__global__ __launch_bounds__(kRowsAtOnce) void k_muon_table(Rows in, int at, int n, Row* rows) {
  if ((int)threadIdx.x < n) rows[at + threadIdx.x] = in.row[threadIdx.x];
}

// --------------------------------------------------------------------- host

int64_t up(int64_t n, int64_t m) { return (n + m - 1) / m * m; }

// A matrix's factors: X [m][n] and X^T [n][m] with m <= n, X^T's next value,
// and the products of X with itself.
struct Shape {
  int64_t rows, cols;
  int64_t m, n, ldm, ldn;  // padded; bytes of rows of m and n elements
  int64_t x, xt[2], square[5], bytes;
  bool tall, wide;  // wide: several steps at once
};

// How many steps go at once.  One step takes 3 m^2 n + m^3 operations (symmetric results half), k at once
// 3 m^2 n + (4 k - 3) m^3: five as 3 + 2 instead take 38 in place of 65 m^3 for n = 4 m (2048 x 8192,
// one matrix: 2.1 ms, one by one 3.0).  Errors of A grow in P A P, where those of X X^T do not: of five steps from 2.2e-6 of the
// result's norm to 3.1e-6 at 512 x 2048 (fp32 arithmetic throughout: 2.8e-6), but from 1.2e-6 to 5.3e-6 at
// 37 x 100, and below 512 latency counts, not operations (one of 256 x 1024 115 us one by one, 117 so).  Where n is little
// more than m it does so above, too: one by one / several at once, 512 x 768 149 / 157 us, 1024 x 1536 255 / 253, 2048 x 2560 954 / 960, 2048 x 3200
// 1075 / 1013, four of these 3387 / 3075.  Three come first, then two, then one at a
// time: once singular values have arrived near 1 errors grow faster (six steps as 3 + 3 1.4e-5).
bool several_at_once(int64_t m, int64_t n) { return m >= 512 && 2 * n >= 3 * m; }
Shape shape_of(int64_t rows, int64_t cols) {
  Shape s = {};
  s.rows = rows;
  s.cols = cols;
  s.tall = rows > cols;
  s.m = up(std::min(rows, cols), kPad);
  s.n = up(std::max(rows, cols), kPad);
  s.ldm = (s.m / kLine | 1) * 128;
  s.ldn = (s.n / kLine | 1) * 128;
  int64_t at = 0;
  auto take = [&](int64_t bytes) {
    const int64_t here = at;
    at += up(bytes, 256);
    return here;
  };
  s.x = take(s.m * s.ldn);
  for (int64_t& t : s.xt) t = take(s.n * s.ldm);
  s.wide = several_at_once(s.m, s.n);
  for (int i = 0; i < (s.wide ? 5 : 2); ++i) s.square[i] = take(s.m * s.ldm);
  s.bytes = at;
  return s;
}

bool is_tiny(int64_t rows, int64_t cols) { return std::min(rows, cols) <= kTinyM && std::max(rows, cols) <= kTinyN; }

// Small matrices, of these sizes at most.
template <typename GT, typename PT, bool MUON>
int32_t launch_tiny(Tiny t, int64_t count, int64_t m, int64_t n, const Source& s, const Last& last, hipStream_t st, std::string* e) {
  t.lines = (int32_t)((n + 2 * kLine - 1) / (2 * kLine) * 2);
  auto go = [&](auto kernel, int mb) {
    auto need = [&](int lines) {
      const int sums = mb == 1 ? kTinyParts<1> - 1 : 3 * (kTinyParts<2> - 1);
      return 32 * mb * lines * 128 + lines * kLine * mb * 128 + 32 * mb * mb * 128 + sums * 4096;
    };
    const int bytes = need(t.lines);
    const int32_t r = allow_lds(reinterpret_cast<const void*>(kernel), need(kTinyN / kLine), e);
    if (r != MTDAO_OK) return r;
    hipLaunchKernelGGL(kernel, dim3((unsigned)count), dim3(kTinyThreads), (size_t)bytes, st, t, s, last);
    return (int32_t)MTDAO_OK;
  };
  return m <= 32 ? go(k_muon_tiny<GT, PT, MUON, 1>, 1) : go(k_muon_tiny<GT, PT, MUON, 2>, 2);
}

// Matrices that go through the products together: runs of one shape in the
// table's order.
struct Run {
  Shape shape;
  int32_t matrix, count;
  int64_t at;  // of the first one's factors in the group's memory
};
struct Group {
  std::vector<Run> runs;
  int64_t bytes = 0, chunks = 0;
};
// Memory that a group's factors may take, unless a single matrix needs more.
constexpr int64_t kGroupBytes = INT64_C(4) << 30;

// Chunks of a matrix's elements, and how many times kChunk they are.
int64_t per_chunk(const Shape& s) { return (s.rows * s.cols + (int64_t)kChunk * kMostChunks - 1) / ((int64_t)kChunk * kMostChunks); }
int64_t chunks_of(const Shape& s) {
  const int64_t each = per_chunk(s) * kChunk;
  return (s.rows * s.cols + each - 1) / each;
}

// shapes: in the table's order, equal ones together, none empty.
// (small ones, at the end, are in no group)
std::vector<Group> groups_of(const std::vector<std::pair<int64_t, int64_t>>& shapes) {
  std::vector<Group> groups;
  for (size_t i = 0; i < shapes.size() && !is_tiny(shapes[i].first, shapes[i].second); ++i) {
    const Shape s = shape_of(shapes[i].first, shapes[i].second);
    const bool same = i > 0 && shapes[i] == shapes[i - 1];
    if (groups.empty() || groups.back().bytes + s.bytes > kGroupBytes || (!same && groups.back().runs.size() == kMostParts) ||
        groups.back().chunks + chunks_of(s) > (1 << 30))
      groups.emplace_back();
    Group& g = groups.back();
    if (!same || g.runs.empty()) g.runs.push_back({s, (int32_t)i, 0, g.bytes});
    g.runs.back().count++;
    g.bytes += s.bytes;
    g.chunks += chunks_of(s);
  }
  return groups;
}

// Tiles of a launch.  Large ones read less of the L2 for each product, small ones keep more
// CUs at work; of those of 64 and 128 two workgroups share a CU.  us with tiles of 64 / 128 / 256:
// 16 matrices of 512 x 512 to 512 x 2048: squares (576 / 160 / 48 tiles) 20 / 22 / 51, A = X X^T (as many) 34 / 52 / 110,
// with X (2960 / 744 / 192) 87 / 67 / 72; four of 2048 x 512: squares (144 / 40 / 16) 9 / 18 / 48,
// A 18 / 41 / 106, with X (1024 / 256 / 64) 29 / 23 / 50; 14 of 2048 x 8192: squares (7392 / 1904 / 504) 504 / 372 / 360,
// A 2916 / 1310 / 1189, with X (57344 / 14336 / 3584) 4822 / 2856 / 2712.
constexpr int kBig = 256, kMid = 128, kLittle = 64;
constexpr int64_t kMostLittle = 1000, kMostMid = 1024;

// A = X X^T of few tiles, up to kFewTiles, and many lines is formed in parts of at least kLeastPart lines, as many as
// occupy the CUs once, and joined: 300 x 8000 396 -> 244 us, 1 x 8192 332 -> 153 us; three of 448 x 4096 (108 tiles) 259 -> 245,
// of 448 x 1024 178 -> 180, one of 1000 x 4000 (136 tiles) 317 either way.
constexpr int64_t kFewTiles = 128, kParts = 256, kLeastPart = 8, kManyLines = 32;
constexpr int64_t kPartialBytes = kParts * kLittle * kLittle * 4;

struct Layout {
  size_t sums, partial, factors, bytes;
};
Layout layout_of(const std::vector<Group>& groups, size_t table_rows) {
  int64_t bytes = 0, chunks = 0;
  for (const Group& g : groups) {
    bytes = std::max(bytes, g.bytes);
    chunks = std::max(chunks, g.chunks);
  }
  Layout l;
  l.sums = up256(table_rows * sizeof(Row));
  l.partial = l.sums + up256((size_t)chunks * sizeof(double));
  l.factors = l.partial + (groups.empty() ? 0 : (size_t)kPartialBytes);
  l.bytes = l.factors + (size_t)bytes;
  return l;
}

// The products of a run, one entry per launch.
//
// A step is X <- P X with P = a I + B, B = b A + c A A.  Steps may be taken several at
// once: X <- Q X with Q = P_k .. P_1, and A = X X^T of the next step from that of the one before as
// P A P, all products of m x m matrices that commute and are symmetric, so that half of
// each is formed.  Q is held as alpha I + R, alpha = a^k: the part that acts on
// the directions far below 1 has no rounding.
std::vector<std::vector<Gemm>> products_of(const Run& run, uint8_t* base, int steps) {
  const Shape& s = run.shape;
  uint8_t* at = base + run.at;
  uint8_t *x = at + s.x, *xt[2] = {at + s.xt[0], at + s.xt[1]}, *gram = at + s.square[0];
  Gemm zero;
  std::memset(&zero, 0, sizeof zero);
  zero.step = s.bytes;
  zero.count = run.count;
  zero.matrix = run.matrix;
  std::vector<std::vector<Gemm>> list;
  // out 2^e = k 2^e a b^T, of factors held with ea and eb; plus() adds k 2^e d.
  auto square = [&](const uint8_t* a, int ea, const uint8_t* b, int eb, uint8_t* out, int e, double k) {
    Gemm g = zero;
    g.a = a;
    g.b = b;
    g.out = out;
    g.rows_a = g.rows_b = (int32_t)s.m;
    g.blocks = (int32_t)(s.m / kLine);
    g.lda = g.ldb = g.ldo = (int32_t)s.ldm;
    g.symmetric = 1;
    g.k0 = (float)std::ldexp(k, e - ea - eb);
    return g;
  };
  auto plus = [](Gemm g, int e, const uint8_t* d, int ed, double k) {
    (g.d1 ? g.k2 : g.k1) = (float)std::ldexp(k, e - ed);
    (g.d1 ? g.d2 : g.d1) = d;
    return g;
  };
  for (int done = 0, turn = 0; done < steps; turn ^= 1) {
    const int now = std::min(!s.wide || done > kMostAtOnce ? 1 : done > 0 ? 2 : kMostAtOnce, steps - done);
    Gemm g = square(x, kX, x, kX, gram, kA, 1.0);
    g.blocks = (int32_t)(s.n / kLine);
    g.lda = g.ldb = (int32_t)s.ldn;
    list.push_back({g});
    uint8_t *poly = at + s.square[1], *r = nullptr, *spare = nullptr, *ap = nullptr;
    if (now > 1) {
      ap = at + s.square[2];
      r = at + s.square[3];
      spare = at + s.square[4];
    }
    double alpha = kCa;
    int er = kB;
    for (int i = 0; i < now; ++i) {
      list.push_back({plus(square(gram, kA, gram, kA, poly, kB, kCc), kB, gram, kA, kCb)});
      if (i == 0) {
        std::swap(poly, r);  // Q = a I + B
        if (now > 1) {
          list.push_back({plus(square(gram, kA, r, kB, ap, kA, 1.0), kA, gram, kA, kCa)});
          list.push_back({plus(square(ap, kA, r, kB, gram, kA, 1.0), kA, ap, kA, kCa)});
        }
        continue;
      }
      // alpha a I + (a R + alpha B + B R)
      list.push_back({plus(plus(square(poly, kB, r, er, spare, kR, 1.0), kR, r, er, kCa), kR, poly, kB, alpha)});
      if (i + 1 < now) {
        list.back().push_back(plus(square(gram, kA, poly, kB, ap, kA, 1.0), kA, gram, kA, kCa));
        list.push_back({plus(square(ap, kA, poly, kB, gram, kA, 1.0), kA, ap, kA, kCa)});
      }
      std::swap(r, spare);
      er = kR;
      alpha *= kCa;
    }
    done += now;
    const bool last = done == steps, flip = last && s.tall;
    Gemm apply = zero;  // X <- alpha X + R X
    apply.a = flip ? xt[turn] : r;
    apply.b = flip ? r : xt[turn];
    apply.lda = apply.ldb = (int32_t)s.ldm;
    apply.ldo = (int32_t)(flip ? s.ldm : s.ldn);
    apply.rows_a = (int32_t)(flip ? s.n : s.m);
    apply.rows_b = (int32_t)(flip ? s.m : s.n);
    apply.blocks = (int32_t)(s.m / kLine);
    const int e = last ? 0 : kX;
    apply.k0 = (float)std::ldexp(1.0, e - er - kX);
    apply = plus(apply, e, flip ? xt[turn] : x, kX, alpha);
    if (last) {
      apply.last = 1;
      apply.rows = s.rows;
      apply.cols = s.cols;
    } else {
      apply.out = x;
      apply.turned = xt[turn ^ 1];
      apply.ldt = (int32_t)s.ldm;
    }
    list.push_back({apply});
  }
  return list;
}

template <typename PT>
int32_t launch_products(Gemms& all, const Last& last, float* partial, hipStream_t st, std::string* e) {
  for (int i = 0; i < all.n; ++i) {
    all.gemm[i].parts = 1;
    all.gemm[i].part_blocks = all.gemm[i].blocks;
  }
  auto count = [&](int tile) {
    int64_t items = 0, turns = 0;
    for (int i = 0; i < all.n; ++i) {
      Gemm& g = all.gemm[i];
      g.tiles_a = (g.rows_a + tile - 1) / tile;
      g.tiles_b = (g.rows_b + tile - 1) / tile;
      g.tiles = g.symmetric ? g.tiles_a * (g.tiles_a + 1) / 2 : g.tiles_a * g.tiles_b;
      g.share = (int32_t)(((int64_t)g.tiles * g.count * g.parts + 7) / 8);
      g.first = (int32_t)turns;
      turns += g.share;
      items += (int64_t)g.tiles * g.count;
    }
    return std::make_pair(items, turns);
  };
  auto go = [&](auto kernel, int tile, int threads, int stages) {
    const int bytes = stages * 2 * tile * 128;
    const int32_t r = allow_lds(reinterpret_cast<const void*>(kernel), bytes, e);
    if (r != MTDAO_OK) return r;
    hipLaunchKernelGGL(kernel, dim3((unsigned)(8 * count(tile).second)), dim3((unsigned)threads), (size_t)bytes, st, all, last);
    return (int32_t)MTDAO_OK;
  };
  const int64_t little = count(kLittle).first;
  int64_t joined = 0;
  if (little <= kFewTiles) {
    float* to = partial;
    for (int i = 0; i < all.n; ++i) {
      Gemm& g = all.gemm[i];
      if (!g.symmetric || g.d1 || g.blocks < kManyLines) continue;
      const int64_t parts = std::min(kParts / little, g.blocks / kLeastPart);
      g.part_blocks = (int32_t)((g.blocks + parts - 1) / parts);
      g.parts = (g.blocks + g.part_blocks - 1) / g.part_blocks;
      if (g.parts == 1) continue;
      g.partial = to;
      to += (int64_t)g.tiles * g.count * g.parts * (kLittle * kLittle);
      joined += (int64_t)g.tiles * g.count;
    }
  }
  if (little <= kMostLittle) {
    const int32_t r = go(k_muon_product<kLittle, 2, 2, 4, PT>, kLittle, 256, 4);
    if (r == MTDAO_OK && joined > 0) hipLaunchKernelGGL(k_muon_join, dim3((unsigned)joined), dim3(256), 0, st, all);
    return r;
  }
  if (count(kMid).first <= kMostMid) return go(k_muon_product<kMid, 2, 2, 2, PT>, kMid, 256, 2);
  return go(k_muon_product<kBig, 2, 4, 2, PT>, kBig, 512, 2);
}

// All the work of a group's matrices.
template <typename GT, typename PT, bool MUON>
int32_t launch_group(const Group& group, Source s, const Last& last, uint8_t* factors, float* partial, int steps, hipStream_t st, std::string* e) {
  Parts parts;
  std::memset(&parts, 0, sizeof parts);
  int64_t chunks = 0, tiles = 0;
  for (const Run& r : group.runs) {
    const Shape& h = r.shape;
    Part& a = parts.part[parts.n++];
    a.natural = factors + r.at + (h.tall ? h.xt[0] : h.x);
    a.turned = factors + r.at + (h.tall ? h.x : h.xt[0]);
    a.ld_natural = (int32_t)(h.tall ? h.ldm : h.ldn);
    a.ld_turned = (int32_t)(h.tall ? h.ldn : h.ldm);
    a.step = h.bytes;
    a.rows = h.rows;
    a.cols = h.cols;
    a.matrix = r.matrix;
    a.count = r.count;
    a.first_chunk = (int32_t)chunks;
    a.chunks = (int32_t)chunks_of(h);
    a.per_chunk = (int32_t)per_chunk(h);
    chunks += (int64_t)a.chunks * r.count;
    a.first_tile = (int32_t)tiles;
    a.tiles_r = (int32_t)((h.tall ? h.n : h.m) / kSplit);
    a.tiles_c = (int32_t)((h.tall ? h.m : h.n) / kSplit);
    tiles += (int64_t)a.tiles_r * a.tiles_c * r.count;
  }
  parts.items = (int32_t)chunks;
  hipLaunchKernelGGL((k_muon_sums<GT, MUON>), grid_of(chunks), dim3(kThreads), 0, st, parts, s);
  parts.items = (int32_t)tiles;
  hipLaunchKernelGGL((k_muon_split<GT, MUON>), grid_of(tiles), dim3(kThreads), 0, st, parts, s);
  std::vector<std::vector<std::vector<Gemm>>> lists;
  size_t most = 0;
  for (const Run& r : group.runs) {
    lists.push_back(products_of(r, factors, steps));
    most = std::max(most, lists.back().size());
  }
  for (size_t i = 0; i < most; ++i) {
    Gemms all;
    std::memset(&all, 0, sizeof all);
    for (const auto& list : lists)
      if (i < list.size())
        for (const Gemm& g : list[i]) all.gemm[all.n++] = g;
    const int32_t r = launch_products<PT>(all, last, partial, st, e);
    if (r != MTDAO_OK) return r;
  }
  return MTDAO_OK;
}

int32_t check_numbers(int32_t steps, double eps, std::string* e) {
  if (steps < 1 || steps > MTDAO_MUON_MAX_STEPS) return fail(e, MTDAO_ERR_INVALID_ARG, "steps %d: 1..%d", steps, MTDAO_MUON_MAX_STEPS);
  if (!(eps >= 0.0) || !std::isfinite(eps)) return fail(e, MTDAO_ERR_INVALID_ARG, "eps=%g must be finite and >= 0", eps);
  return MTDAO_OK;
}
int32_t check_sides(int64_t rows, int64_t cols, int i, std::string* e) {
  if (rows < 0 || cols < 0) return fail(e, MTDAO_ERR_INVALID_ARG, "rows or cols of matrix %d < 0", i);
  if (std::min(rows, cols) > MTDAO_MUON_MAX_SIDE || std::max(rows, cols) > (INT64_C(1) << 20))
    return fail(e, MTDAO_ERR_INVALID_ARG, "matrix %d is %lld x %lld: its smaller side is at most %d, its larger one 2^20", i, (long long)rows, (long long)cols,
                MTDAO_MUON_MAX_SIDE);
  return MTDAO_OK;
}
int32_t check_type(int32_t dtype, const char* name, std::string* e) {
  if (dtype != MTDAO_F32 && dtype != MTDAO_BF16) return fail(e, MTDAO_ERR_INVALID_ARG, "%s must be F32(0) or BF16(1)", name);
  return MTDAO_OK;
}
int32_t check_workspace(const void* workspace, size_t given, size_t need, std::string* e) {
  if (!workspace || given < need)
    return fail(e, MTDAO_ERR_WORKSPACE, "workspace of %zu bytes required, %zu given", need, workspace ? given : (size_t)0);
  if (!aligned_to(workspace, 256)) return fail(e, MTDAO_ERR_ALIGN, "workspace is not 256-byte aligned");
  return MTDAO_OK;
}

int32_t validate(const mtdao_muon_config* c, const mtdao_muon_matrix* t, std::string* e) {
  if (!c || !t) return fail(e, MTDAO_ERR_INVALID_ARG, "config or matrices is NULL");
  int32_t r = check_type(c->param_dtype, "param_dtype", e);
  if (r == MTDAO_OK) r = check_type(c->grad_dtype, "grad_dtype", e);
  if (r == MTDAO_OK) r = check_numbers(c->steps, c->eps, e);
  if (r != MTDAO_OK) return r;
  if (c->n_matrices < 1 || c->n_matrices > (1 << 20)) return fail(e, MTDAO_ERR_INVALID_ARG, "n_matrices %d: 1..2^20", c->n_matrices);
  if (!(c->momentum >= 0.0 && c->momentum < 1.0)) return fail(e, MTDAO_ERR_INVALID_ARG, "momentum=%g: in [0,1)", c->momentum);
  for (int i = 0; i < c->n_matrices; ++i) {
    r = check_sides(t[i].rows, t[i].cols, i, e);
    if (r != MTDAO_OK) return r;
    if (!(t[i].weight_decay >= 0.0) || !std::isfinite((float)t[i].weight_decay))
      return fail(e, MTDAO_ERR_INVALID_ARG, "weight_decay of matrix %d must be finite and >= 0", i);
    if (!std::isfinite((float)t[i].factor)) return fail(e, MTDAO_ERR_INVALID_ARG, "factor of matrix %d is not finite", i);
  }
  return MTDAO_OK;
}

struct Written {
  uintptr_t lo, hi;
};

// Gradients are read after the momenta are written.
int32_t check_grad(const mtdao_muon_config& c, int i, int64_t numel, const void* g, const std::vector<Written>& written, std::string* e) {
  if (numel == 0) return MTDAO_OK;
  if (!g) return fail(e, MTDAO_ERR_INVALID_ARG, "g of matrix %d is NULL", i);
  if (!aligned_to(g, (uintptr_t)esize(c.grad_dtype))) return fail(e, MTDAO_ERR_ALIGN, "g of matrix %d is not aligned to its element", i);
  const uintptr_t lo = (uintptr_t)g, hi = lo + (uintptr_t)(numel * esize(c.grad_dtype));
  auto w = std::upper_bound(written.begin(), written.end(), lo, [](uintptr_t at, const Written& r) { return at < r.hi; });
  if (w != written.end() && w->lo < hi) return fail(e, MTDAO_ERR_INVALID_ARG, "g of matrix %d overlaps parameters or momenta", i);
  return MTDAO_OK;
}

int32_t check_pointers(const mtdao_muon_config& c, const mtdao_muon_matrix* t, std::vector<Written>& written, std::string* e) {
  for (int i = 0; i < c.n_matrices; ++i) {
    const int64_t numel = t[i].rows * t[i].cols;
    if (numel == 0) continue;
    if (!t[i].p || !t[i].m) return fail(e, MTDAO_ERR_INVALID_ARG, "p or m of matrix %d is NULL", i);
    if (!aligned_to(t[i].p, (uintptr_t)esize(c.param_dtype)) || !aligned_to(t[i].m, 4))
      return fail(e, MTDAO_ERR_ALIGN, "p or m of matrix %d is not aligned to its element", i);
    written.push_back({(uintptr_t)t[i].p, (uintptr_t)t[i].p + (uintptr_t)(numel * esize(c.param_dtype))});
    written.push_back({(uintptr_t)t[i].m, (uintptr_t)t[i].m + (uintptr_t)(numel * 4)});
  }
  std::sort(written.begin(), written.end(), [](const Written& x, const Written& y) { return x.lo < y.lo; });
  for (size_t k = 1; k < written.size(); ++k)
    if (written[k].lo < written[k - 1].hi) return fail(e, MTDAO_ERR_INVALID_ARG, "parameters or momenta of the matrices overlap");
  for (int i = 0; i < c.n_matrices; ++i) {
    const int32_t r = check_grad(c, i, t[i].rows * t[i].cols, t[i].g, written, e);
    if (r != MTDAO_OK) return r;
  }
  return MTDAO_OK;
}

// Matrices in the table's order (shapes together, small ones at the end, none empty): their numbers.
std::vector<int> order_of(const mtdao_muon_config& c, const mtdao_muon_matrix* t) {
  std::vector<int> order;
  for (int i = 0; i < c.n_matrices; ++i)
    if (t[i].rows > 0 && t[i].cols > 0) order.push_back(i);
  std::stable_sort(order.begin(), order.end(), [&](int a, int b) {
    const bool ta = is_tiny(t[a].rows, t[a].cols), tb = is_tiny(t[b].rows, t[b].cols);
    return ta != tb ? tb : std::make_pair(t[a].rows * t[a].cols, t[a].rows) > std::make_pair(t[b].rows * t[b].cols, t[b].rows);
  });
  return order;
}
std::vector<Group> groups_of(const std::vector<int>& order, const mtdao_muon_matrix* t) {
  std::vector<std::pair<int64_t, int64_t>> shapes;
  for (int i : order) shapes.push_back({t[i].rows, t[i].cols});
  return groups_of(shapes);
}
std::vector<Group> groups_of(int64_t batch, int64_t rows, int64_t cols) {
  return groups_of(std::vector<std::pair<int64_t, int64_t>>((size_t)(rows > 0 && cols > 0 ? batch : 0), {rows, cols}));
}

int32_t check_batch(int64_t batch, int64_t rows, int64_t cols, std::string* e) {
  if (batch < 0 || batch > (1 << 20)) return fail(e, MTDAO_ERR_INVALID_ARG, "batch %lld: 0..2^20", (long long)batch);
  return check_sides(rows, cols, 0, e);
}

}  // namespace

struct mtdao_muon {
  mtdao_muon_config cfg;
  std::vector<int64_t> numel;       // of every matrix
  std::vector<int> order;
  std::vector<Row> rows;            // the table
  std::vector<Written> written;
  std::vector<Group> groups;
  size_t tiny = 0;                  // small matrices, and their largest sides
  int64_t tiny_m = 0, tiny_n = 0;
  Layout layout;
  char* workspace = nullptr;
  std::string err;
};

namespace {
int32_t write_table(mtdao_muon* h, std::string* e, hipStream_t st) {
  for (size_t at = 0; at < h->rows.size(); at += kRowsAtOnce) {
    Rows in;
    std::memset(&in, 0, sizeof in);
    const int n = (int)std::min<size_t>(kRowsAtOnce, h->rows.size() - at);
    std::copy_n(h->rows.begin() + at, n, in.row);
    hipLaunchKernelGGL(k_muon_table, dim3(1), dim3(kRowsAtOnce), 0, st, in, (int)at, n, reinterpret_cast<Row*>(h->workspace));
  }
  return hip_check(e, hipGetLastError(), "mtdao_muon table launch");
}
}  // namespace

extern "C" {

int32_t mtdao_orthogonalize_workspace_bytes(int64_t batch, int64_t rows, int64_t cols, size_t* bytes) try {
  const int32_t r = check_batch(batch, rows, cols, &g_err);
  if (r != MTDAO_OK) return r;
  if (!bytes) return fail(&g_err, MTDAO_ERR_INVALID_ARG, "bytes is NULL");
  const std::vector<Group> groups = groups_of(batch, rows, cols);
  *bytes = groups.empty() ? 0 : layout_of(groups, 0).bytes;  // (small matrices need none)
  return MTDAO_OK;
} catch (const std::bad_alloc&) {
  return fail(&g_err, MTDAO_ERR_WORKSPACE, "out of host memory");
}

int32_t mtdao_orthogonalize(const void* x, int32_t dtype, int64_t batch, int64_t rows, int64_t cols, void* out, int32_t out_dtype,
                            int32_t steps, double eps, void* workspace, size_t workspace_bytes, void* hip_stream) try {
  std::string* e = &g_err;
  int32_t r = check_batch(batch, rows, cols, e);
  if (r == MTDAO_OK) r = check_type(dtype, "dtype", e);
  if (r == MTDAO_OK) r = check_type(out_dtype, "out_dtype", e);
  if (r == MTDAO_OK) r = check_numbers(steps, eps, e);
  if (r != MTDAO_OK) return r;
  if (batch == 0 || rows == 0 || cols == 0) return MTDAO_OK;
  if (!x || !out) return fail(e, MTDAO_ERR_INVALID_ARG, "x or out is NULL");
  if (!aligned_to(x, (uintptr_t)esize(dtype)) || !aligned_to(out, (uintptr_t)esize(out_dtype)))
    return fail(e, MTDAO_ERR_ALIGN, "x or out is not aligned to its element");
  const int64_t numel = batch * rows * cols;
  // (matrices go group by group, so a later one's x may not lie under an earlier one's result)
  if (overlap(x, numel * esize(dtype), out, numel * esize(out_dtype)) && (x != out || dtype != out_dtype))
    return fail(e, MTDAO_ERR_INVALID_ARG, "out overlaps x");
  hipStream_t st = reinterpret_cast<hipStream_t>(hip_stream);
  const Last last = {nullptr, out, 0.0f};
  auto with = [&](auto go) {
    if (dtype == MTDAO_F32 && out_dtype == MTDAO_F32) return go(float{}, float{});
    if (dtype == MTDAO_F32) return go(float{}, bf16_t{});
    if (out_dtype == MTDAO_F32) return go(bf16_t{}, float{});
    return go(bf16_t{}, bf16_t{});
  };
  if (is_tiny(rows, cols)) {
    RoctxRange range("mtdao_orthogonalize %lld x %lld x %lld", (long long)batch, (long long)rows, (long long)cols);
    const Source s = {nullptr, x, nullptr, 0.0f, 0, eps};
    r = with([&](auto g, auto p) {
      return launch_tiny<decltype(g), decltype(p), false>({0, 0, rows, cols, steps}, batch, std::min(rows, cols), std::max(rows, cols), s, last, st, e);
    });
    return r != MTDAO_OK ? r : hip_check(e, hipGetLastError(), "mtdao_orthogonalize launch");
  }
  const std::vector<Group> groups = groups_of(batch, rows, cols);
  const Layout l = layout_of(groups, 0);
  r = check_workspace(workspace, workspace_bytes, l.bytes, e);
  if (r != MTDAO_OK) return r;
  char* w = static_cast<char*>(workspace);
  RoctxRange range("mtdao_orthogonalize %lld x %lld x %lld", (long long)batch, (long long)rows, (long long)cols);
  const Source s = {nullptr, x, reinterpret_cast<double*>(w + l.sums), 0.0f, 0, eps};
  for (const Group& g : groups) {
    r = with([&](auto gt, auto pt) {
      return launch_group<decltype(gt), decltype(pt), false>(g, s, last, reinterpret_cast<uint8_t*>(w + l.factors), reinterpret_cast<float*>(w + l.partial), steps, st, e);
    });
    if (r != MTDAO_OK) return r;
  }
  return hip_check(e, hipGetLastError(), "mtdao_orthogonalize launch");
} catch (const std::bad_alloc&) {
  return fail(&g_err, MTDAO_ERR_WORKSPACE, "out of host memory");
}

int32_t mtdao_muon_workspace_bytes(const mtdao_muon_config* cfg, const mtdao_muon_matrix* matrices, size_t* bytes) try {
  const int32_t r = validate(cfg, matrices, &g_err);
  if (r != MTDAO_OK) return r;
  if (!bytes) return fail(&g_err, MTDAO_ERR_INVALID_ARG, "bytes is NULL");
  const std::vector<int> order = order_of(*cfg, matrices);
  *bytes = layout_of(groups_of(order, matrices), order.size()).bytes;
  return MTDAO_OK;
} catch (const std::bad_alloc&) {
  return fail(&g_err, MTDAO_ERR_WORKSPACE, "out of host memory");
}

int32_t mtdao_muon_init(const mtdao_muon_config* cfg, const mtdao_muon_matrix* matrices, void* workspace, size_t workspace_bytes,
                        void* hip_stream, mtdao_muon** out) try {
  int32_t r = validate(cfg, matrices, &g_err);
  if (r != MTDAO_OK) return r;
  if (!out) return fail(&g_err, MTDAO_ERR_INVALID_ARG, "out is NULL");
  std::vector<Written> written;
  r = check_pointers(*cfg, matrices, written, &g_err);
  if (r != MTDAO_OK) return r;
  struct Owned {
    mtdao_muon* h = new mtdao_muon();
    ~Owned() { delete h; }
  } own;
  mtdao_muon* h = own.h;
  h->cfg = *cfg;
  h->order = order_of(*cfg, matrices);
  h->groups = groups_of(h->order, matrices);
  h->layout = layout_of(h->groups, h->order.size());
  if (h->layout.bytes > 0) {
    r = check_workspace(workspace, workspace_bytes, h->layout.bytes, &g_err);
    if (r != MTDAO_OK) return r;
  }
  h->workspace = static_cast<char*>(workspace);
  h->written = std::move(written);
  for (int i = 0; i < cfg->n_matrices; ++i) h->numel.push_back(matrices[i].rows * matrices[i].cols);
  for (int i : h->order) {
    const mtdao_muon_matrix& a = matrices[i];
    h->rows.push_back({a.p, a.g, a.m, (float)a.weight_decay, (float)a.factor, (int32_t)a.rows, (int32_t)a.cols});
    if (is_tiny(a.rows, a.cols)) {
      h->tiny++;
      h->tiny_m = std::max(h->tiny_m, std::min(a.rows, a.cols));
      h->tiny_n = std::max(h->tiny_n, std::max(a.rows, a.cols));
    }
  }
  RoctxRange range("mtdao_muon_init matrices=%d", cfg->n_matrices);
  r = write_table(h, &g_err, reinterpret_cast<hipStream_t>(hip_stream));
  if (r != MTDAO_OK) return r;
  g_err.clear();
  *out = h;
  own.h = nullptr;
  return MTDAO_OK;
} catch (const std::bad_alloc&) {
  return fail(&g_err, MTDAO_ERR_WORKSPACE, "out of host memory");
}

int32_t mtdao_muon_set_grads(mtdao_muon* h, const void* const* grads, void* hip_stream) {
  if (!h) return fail(&g_err, MTDAO_ERR_INVALID_ARG, "handle is NULL");
  if (!grads) return fail(&h->err, MTDAO_ERR_INVALID_ARG, "grads is NULL");
  for (int i = 0; i < h->cfg.n_matrices; ++i) {
    const int32_t r = check_grad(h->cfg, i, h->numel[i], grads[i], h->written, &h->err);
    if (r != MTDAO_OK) return r;
  }
  RoctxRange range("mtdao_muon_set_grads matrices=%d", h->cfg.n_matrices);
  for (size_t k = 0; k < h->order.size(); ++k) h->rows[k].g = grads[h->order[k]];
  return write_table(h, &h->err, reinterpret_cast<hipStream_t>(hip_stream));
}

int32_t mtdao_muon_step(mtdao_muon* h, double lr, void* hip_stream) try {
  if (!h) return fail(&g_err, MTDAO_ERR_INVALID_ARG, "handle is NULL");
  if (!std::isfinite((float)lr)) return fail(&h->err, MTDAO_ERR_INVALID_ARG, "lr is not finite");
  const mtdao_muon_config& c = h->cfg;
  hipStream_t st = reinterpret_cast<hipStream_t>(hip_stream);
  RoctxRange range("mtdao_muon_step matrices=%d", c.n_matrices);
  char* w = h->workspace;
  const Row* rows = reinterpret_cast<const Row*>(w);
  const Source s = {rows, nullptr, reinterpret_cast<double*>(w + h->layout.sums), (float)c.momentum, c.nesterov != 0, c.eps};
  const Last last = {rows, nullptr, (float)lr};
  uint8_t* factors = reinterpret_cast<uint8_t*>(w + h->layout.factors);
  float* partial = reinterpret_cast<float*>(w + h->layout.partial);
  auto with = [&](auto go) {
    if (c.param_dtype == MTDAO_F32 && c.grad_dtype == MTDAO_F32) return go(float{}, float{});
    if (c.param_dtype == MTDAO_F32) return go(bf16_t{}, float{});
    if (c.grad_dtype == MTDAO_F32) return go(float{}, bf16_t{});
    return go(bf16_t{}, bf16_t{});
  };
  int32_t r = MTDAO_OK;
  for (const Group& g : h->groups) {
    r = with([&](auto gt, auto pt) { return launch_group<decltype(gt), decltype(pt), true>(g, s, last, factors, partial, c.steps, st, &h->err); });
    if (r != MTDAO_OK) return r;
  }
  if (h->tiny > 0) {
    r = with([&](auto gt, auto pt) {
      return launch_tiny<decltype(gt), decltype(pt), true>({(int32_t)(h->rows.size() - h->tiny), 0, 0, 0, c.steps}, (int64_t)h->tiny, h->tiny_m, h->tiny_n, s, last,
                                                           st, &h->err);
    });
    if (r != MTDAO_OK) return r;
  }
  return hip_check(&h->err, hipGetLastError(), "mtdao_muon_step launch");
} catch (const std::bad_alloc&) {
  return fail(h ? &h->err : &g_err, MTDAO_ERR_WORKSPACE, "out of host memory");
}

const char* mtdao_muon_last_error(const mtdao_muon* h) { return h ? h->err.c_str() : g_err.c_str(); }

void mtdao_muon_destroy(mtdao_muon* h) { delete h; }

}  // extern "C"
