// Matrices in 8-bit floating point with a scale per block of 128, and their
// product (include/mtdao_ops.h).

#include <hip/hip_runtime.h>

#include <algorithm>
#include <mutex>
#include <new>
#include <set>
#include <string>
#include <type_traits>
#include <utility>

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
  int64_t rows, ld, scale_rows;  // scale_rows: rows of scales
  int64_t scale_ld;              // bytes from four blocks' scales to the next four's: 4 scale_rows
  int32_t blocks;                // blocks of a row
};
__device__ __forceinline__ uint8_t* scale_at(const Mat& m, int64_t scale_row, int block) {
  return m.scales + (block >> 2) * m.scale_ld + scale_row * 4 + (block & 3);
}

// --------------------------------------------------------------- quantizers

constexpr int kThreads = 256;
constexpr int kE = 8;  // elements of a thread's vector: 16 threads hold a block

// Both quantizers are bound by HBM: an element is read once, and a byte written
// for each orientation.

// Blocks along the rows: four of each of four rows a workgroup, a row a wave; a
// block's largest value is found by its sixteen lanes.  16384 x 8192 bf16: 5.6 TB/s.
template <typename T>
__global__ __launch_bounds__(kThreads) void k_quantize8_rows(const T* x, int64_t ld, int64_t cols, int groups, int fours, Mat q) {
  const unsigned in_x = blockIdx.x / (unsigned)groups;  // of `fours` along x
  const int64_t row = ((int64_t)blockIdx.y * fours + in_x) * 4 + threadIdx.x / 64;
  const int kb = (int)(blockIdx.x - in_x * groups) * 4 + (int)threadIdx.x % 64 / 16, e = kb * kBlock8 + (int)(threadIdx.x % 16) * kE;
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
  for (int t = 0; t < kE; ++t) most = max_abs(most, a[t]);
  if (is_infinite(most)) {
    most = 0.0f;
#pragma unroll
    for (int t = 0; t < kE; ++t) most = fmaxf(most, finite_abs(a[t]));
  }
  const uint32_t byte = live ? scale_byte(max16(most)) : 127u;
  const float inv = inverse_scale_of(byte);
#pragma unroll
  for (int t = 0; t < kE; ++t) a[t] *= inv;
  if (live) {
    uint2 c = {codes_of(a[0], a[1], a[2], a[3]), codes_of(a[4], a[5], a[6], a[7])};
    *reinterpret_cast<uint2*>(q.codes + row * q.ld + e) = c;
  }
  if (row < q.rows && threadIdx.x % 16 == 0) *scale_at(q, row, kb) = (uint8_t)byte;
}

// A tile of 128 x 128: a thread holds four rows of eight columns, so that it
// has four consecutive bytes of each transposed row.  SQUARE: one scale for
// the tile; else blocks along the rows for q, along the columns for qt.  qt
// goes through LDS to be written in whole lines.  16384 x 8192 bf16 both ways:
// 107 us, 5.0 TB/s; the transposed one alone 4.9 TB/s.
// A launch takes one matrix, or two of as many rows one beside the other.
struct Quantized {
  const void* x;
  int64_t ld, cols;
  Mat q, qt;      // codes NULL: not wanted
  int32_t tiles;  // across
};
constexpr int kTileThreads = 512;
template <typename T, bool SQUARE>
__global__ __launch_bounds__(kTileThreads) void k_quantize8_tile(Quantized one, Quantized two, int64_t rows) {
  const bool first = (int)blockIdx.x < one.tiles;
  const T* x = reinterpret_cast<const T*>(first ? one.x : two.x);
  const int64_t ld = first ? one.ld : two.ld, cols = first ? one.cols : two.cols;
  const Mat q = first ? one.q : two.q, qt = first ? one.qt : two.qt;
  const int tile = first ? (int)blockIdx.x : (int)blockIdx.x - one.tiles, tiles = first ? one.tiles : two.tiles;
  constexpr int kRows = 4, kWaves = kTileThreads / 64;
  __shared__ __attribute__((aligned(16))) uint8_t turned[kBlock8 * kBlock8];
  __shared__ __attribute__((aligned(16))) float most[kWaves][kBlock8];
  __shared__ __attribute__((aligned(8))) uint8_t bytes_of[kBlock8];
  const int c8 = (int)(threadIdx.x % 16) * kE, r4 = (int)(threadIdx.x / 16) * kRows, wave = threadIdx.x / 64;
  const int64_t row0 = (int64_t)blockIdx.y * kBlock8, col0 = (int64_t)tile * kBlock8;
  const int64_t in_cols = cols - col0 - c8, in_rows = rows - row0 - r4;
  const int nc = in_cols < 0 ? 0 : in_cols > kE ? kE : (int)in_cols;
  float a[kRows][kE];
#pragma unroll
  for (int i = 0; i < kRows; ++i) {
    if (i < in_rows && nc > 0) {
      load_some<kE>(x + (row0 + r4 + i) * ld + col0 + c8, nc, a[i]);
    } else {
#pragma unroll
      for (int t = 0; t < kE; ++t) a[i][t] = 0.0f;
    }
  }
  float rmax[kRows], cmax[kE], all = 0.0f;
#pragma unroll
  for (int t = 0; t < kE; ++t) cmax[t] = 0.0f;
#pragma unroll
  for (int i = 0; i < kRows; ++i) {
    rmax[i] = 0.0f;
#pragma unroll
    for (int t = 0; t < kE; ++t) {
      rmax[i] = max_abs(rmax[i], a[i][t]);
      cmax[t] = max_abs(cmax[t], a[i][t]);
    }
    all = fmaxf(all, rmax[i]);
  }
  if (is_infinite(all)) {
    all = 0.0f;
#pragma unroll
    for (int t = 0; t < kE; ++t) cmax[t] = 0.0f;
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
      rmax[i] = 0.0f;
#pragma unroll
      for (int t = 0; t < kE; ++t) {
        rmax[i] = fmaxf(rmax[i], finite_abs(a[i][t]));
        cmax[t] = fmaxf(cmax[t], finite_abs(a[i][t]));
      }
      all = fmaxf(all, rmax[i]);
    }
  }
  uint32_t row_byte[kRows], col_byte[kE];
  if constexpr (SQUARE) {
    all = max_with32(max32(all));
    if (threadIdx.x % 64 == 0) most[0][wave] = all;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kWaves; ++w) all = fmaxf(all, most[0][w]);
    const uint32_t byte = scale_byte(all);
#pragma unroll
    for (int i = 0; i < kRows; ++i) row_byte[i] = byte;
#pragma unroll
    for (int t = 0; t < kE; ++t) col_byte[t] = byte;
  } else {
#pragma unroll
    for (int i = 0; i < kRows; ++i) row_byte[i] = scale_byte(max16(rmax[i]));
    // columns: the four rows of threads of a wave, then the waves
#pragma unroll
    for (int t = 0; t < kE; ++t) cmax[t] = max_with32(max_with16(cmax[t]));
    if (threadIdx.x % 64 < 16) {
#pragma unroll
      for (int t = 0; t < kE; t += 4)
        *reinterpret_cast<float4*>(&most[wave][c8 + t]) = float4{cmax[t], cmax[t + 1], cmax[t + 2], cmax[t + 3]};
    }
    __syncthreads();
    if (threadIdx.x < kBlock8) {
      float m = 0.0f;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) m = fmaxf(m, most[w][threadIdx.x]);
      bytes_of[threadIdx.x] = (uint8_t)scale_byte(m);
    }
    __syncthreads();
    const uint2 b = *reinterpret_cast<const uint2*>(bytes_of + c8);
#pragma unroll
    for (int t = 0; t < kE; ++t) col_byte[t] = ((t < 4 ? b.x : b.y) >> 8 * (t & 3)) & 255u;
  }
  if (q.codes) {
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
      const float inv = inverse_scale_of(row_byte[i]);
      float s[kE];
#pragma unroll
      for (int t = 0; t < kE; ++t) s[t] = a[i][t] * inv;
      if (i < in_rows) {
        uint2 c = {codes_of(s[0], s[1], s[2], s[3]), codes_of(s[4], s[5], s[6], s[7])};
        *reinterpret_cast<uint2*>(q.codes + (row0 + r4 + i) * q.ld + col0 + c8) = c;
      }
    }
    // (the last block's thread writes the unused bytes of its four too)
    const int past = tile + 1 == tiles ? (tile & ~3) + 4 : tile + 1;
    if constexpr (SQUARE) {
      if (threadIdx.x == 0)
        for (int k = tile; k < past; ++k) *scale_at(q, blockIdx.y, k) = k == tile ? (uint8_t)row_byte[0] : 127;
    } else if (threadIdx.x % 16 == 0) {
#pragma unroll
      for (int i = 0; i < kRows; ++i)
        if (i < in_rows)
          for (int k = tile; k < past; ++k) *scale_at(q, row0 + r4 + i, k) = k == tile ? (uint8_t)row_byte[i] : 127;
    }
  }
  if (qt.codes) {
    // row c of turned: its 16-byte chunk k at place k ^ c / 8 % 8, which
    // spreads a wave's writes over half of the banks
    const int chunk = r4 / 16, in_chunk = r4 % 16;
#pragma unroll
    for (int t = 0; t < kE; ++t) {
      const float inv = inverse_scale_of(col_byte[t]);
      float s[kRows];
#pragma unroll
      for (int i = 0; i < kRows; ++i) s[i] = a[i][t] * inv;
      *reinterpret_cast<uint32_t*>(turned + (c8 + t) * kBlock8 + ((chunk ^ (c8 / 8 & 7)) << 4) + in_chunk) =
          codes_of(s[0], s[1], s[2], s[3]);
    }
    const int past = blockIdx.y + 1 == gridDim.y ? (blockIdx.y & ~3u) + 4 : blockIdx.y + 1;
    if constexpr (SQUARE) {
      if (threadIdx.x == 0)
        for (int k = blockIdx.y; k < past; ++k) *scale_at(qt, tile, k) = k == (int)blockIdx.y ? (uint8_t)col_byte[0] : 127;
    } else if (threadIdx.x < 16) {
#pragma unroll
      for (int t = 0; t < kE; ++t)
        if (t < nc)
          for (int k = blockIdx.y; k < past; ++k) *scale_at(qt, col0 + c8 + t, k) = k == (int)blockIdx.y ? (uint8_t)col_byte[t] : 127;
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kBlock8 * 8 / kTileThreads; ++k) {
      const int at = k * kTileThreads + (int)threadIdx.x, r = at / 8, c = at % 8;
      if (col0 + r < cols)
        *reinterpret_cast<uint4*>(qt.codes + (col0 + r) * qt.ld + row0 + c * 16) =
            *reinterpret_cast<const uint4*>(turned + r * kBlock8 + ((c ^ (r / 8 & 7)) << 4));
    }
  }
}

// ------------------------------------------------------------------ product
//
// Every matrix instruction takes 32 x 64 codes of each side, half a block, and
// their scales: as these are powers of two in the instruction's own format,
// sums stay in its accumulators from the first block to the last.  Which
// 16-byte chunks of a block a lane holds is free as long as both sides agree,
// since they share one scale.  Rows of b go in as the instruction's rows, so
// that a lane ends with sixteen consecutive columns of a row of c.
//
// Within a group of eight products, neighbours in a row, the 8-bit instructions
// drop what lies more than 13 bits below the largest one (measured: 65536 + 4 gives
// 65536, 65536 + 8 does not, in the instruction with scales and the one without;
// 4 in the next group stays), which leaves sums 1.3e-5
// (normal values) to 4e-5 (outlier columns) off in relative norm.  For a bf16
// c that is a fortieth of its rounding, 1.7e-3, and rate counts for more.  An fp32 c is formed by bf16
// instructions instead, at half their rate: codes times scales are bf16
// values, and their products are summed in fp32.

typedef int v8i __attribute__((ext_vector_type(8)));
typedef int v4i __attribute__((ext_vector_type(4)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef float v16f __attribute__((ext_vector_type(16)));
typedef __bf16 v2bf __attribute__((ext_vector_type(2)));
typedef __bf16 v8bf __attribute__((ext_vector_type(8)));

struct Product {
  Mat a, b;
  void* c;
  int64_t ldc;
  int32_t a_scale_shift, b_scale_shift;  // rows of a scale: 1 << shift
  int32_t accumulate, tiles_m, tiles_n, group;
  int32_t splits, split_blocks;  // parts of the contraction, and their blocks
  float* partial;                // [splits][rows of a][rows of b] with more than one part
};

// A 128-byte row in LDS: each of its eight 16-byte chunks is at the place that its
// number and the row's key give, by an exclusive or.  A 16-byte read of a wave takes 16 lanes at
// once, which have to lie in different ones of the 16 such places of the 64
// banks: two rows of eight, told apart by the row's last bit, so the key has
// the next three.  (With the last three bits as the key half of the reads'
// cycles were conflicts.)
__device__ __forceinline__ int row_key(int row) { return (row >> 1) & 7; }

// The row of b's fragment that the instruction's row r takes: results of a lane
// are rows 8 q + 4 h + t, so these are sixteen consecutive columns of c.
__device__ __forceinline__ int row_of_b(int r) { return ((r >> 2) & 1) * 16 + (r >> 3) * 4 + (r & 3); }

// Eight codes times their scale, as bf16: exact down to bf16's smallest values.
__device__ __forceinline__ v8bf widened(int w0, int w1, float scale) {
  v8bf o;
  const int w[2] = {w0, w1};
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const v2bf lo = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((unsigned)w[k], scale, false);
    const v2bf hi = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((unsigned)w[k], scale, true);
    o[4 * k] = lo[0];
    o[4 * k + 1] = lo[1];
    o[4 * k + 2] = hi[0];
    o[4 * k + 3] = hi[1];
  }
  return o;
}

__device__ __forceinline__ __amdgpu_buffer_rsrc_t buffer_of(const uint8_t* p, int64_t bytes) {
  const int64_t most = INT64_C(0x7fffffff);
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(p), 0, (int)(bytes < most ? bytes : most), 0x00027000);
}

// Every wave of the workgroup has come here; nothing is moved across.
__device__ __forceinline__ void meet() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_sched_barrier(0);
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_sched_barrier(0);
  asm volatile("" ::: "memory");
}
// This wave's loads (global memory to registers or LDS; LDS to registers)
// have arrived, but for the last LEFT of them.
template <int LEFT = 0>
__device__ __forceinline__ void loads_landed() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(0x0f70 | (LEFT & 15) | (LEFT >> 4) << 14);  // vmcnt(LEFT)
  asm volatile("" ::: "memory");
}
__device__ __forceinline__ void reads_landed() { __builtin_amdgcn_s_waitcnt(0xc07f); }  // lgkmcnt(0)

// Tile t of c's tiles in the order in which they are worked on: groups of
// p.group tile rows, down the rows first, so that tiles in work at one time
// share their rows of a and b in the L2.
struct Place {
  int64_t row0, col0;
};
template <int BM, int BN>
__device__ __forceinline__ Place place_of(const Product& p, int t) {
  const int group = t / (p.group * p.tiles_n), in_group = t - group * p.group * p.tiles_n;
  const int rows_here = p.tiles_m - group * p.group < p.group ? p.tiles_m - group * p.group : p.group;
  return {(int64_t)(group * p.group + in_group % rows_here) * BM, (int64_t)(in_group / rows_here) * BN};
}

// A step of half a block: what its matrix instructions take of a row, in a
// lane.  8-bit instructions: one step of two 16-byte chunks (the half block over
// the two halves of the wave); bf16 instructions: two steps of one chunk.
template <bool WIDE>
struct Step8 {
  static constexpr int kSteps = WIDE ? 2 : 1;
  using Fragment = std::conditional_t<WIDE, v4i, v8i>;
  // `row`: where the lane's first chunk is; the second is an exclusive or away.
  static __device__ __forceinline__ Fragment read(const uint8_t* lds, int row, int offset, int step) {
    if constexpr (WIDE) {
      return *reinterpret_cast<const v4i*>(lds + offset + (row ^ step * 16));
    } else {
      const v4i a = *reinterpret_cast<const v4i*>(lds + offset + row);
      const v4i b = *reinterpret_cast<const v4i*>(lds + offset + (row ^ 16));
      return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
    }
  }
  // The products of a step, into acc.  between(t) is called after parts of the
  // instructions, t = 0 .. calls - 1: what it issues goes out while the matrix
  // cores work.
  template <int MI, int NI>
  static constexpr int calls = WIDE ? 2 * MI : MI * NI;
  template <int MI, int NI, typename F>
  static __device__ __forceinline__ void multiply(const Fragment (&fa)[MI], const Fragment (&fb)[NI], const uint32_t (&ea)[MI],
                                                  const uint32_t (&eb)[NI], v16f (&acc)[MI][NI], F&& between) {
    if constexpr (!WIDE) {
#pragma unroll
      for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int j = 0; j < NI; ++j) {
          acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(fb[j], fa[i], acc[i][j], 0, 0, 0, eb[j], 0, ea[i]);
          between(i * NI + j);
        }
    } else {
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        v8bf wb[NI];
#pragma unroll
        for (int j = 0; j < NI; ++j) wb[j] = widened(fb[j][2 * k], fb[j][2 * k + 1], scale_of(eb[j] & 255u));
#pragma unroll
        for (int i = 0; i < MI; ++i) {
          const v8bf wa = widened(fa[i][2 * k], fa[i][2 * k + 1], scale_of(ea[i] & 255u));
#pragma unroll
          for (int j = 0; j < NI; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(wb[j], wa, acc[i][j], 0, 0, 0);
          between(k * MI + i);
        }
      }
    }
    // (without a use here the instructions would be moved past the next barrier)
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
      for (int j = 0; j < NI; ++j) asm volatile("" : "+v"(acc[i][j]));
  }
};

// Results to c, by way of the wave's own part of LDS: ROWS rows of BYTES bytes
// (64 or 128), of which BYTES / 16 lanes then store one.
template <int BYTES>
__device__ __forceinline__ uint8_t* staged(uint8_t* own, int row, int chunk) {
  return own + row * BYTES + ((chunk ^ ((row * BYTES / 256) & (BYTES / 16 - 1))) << 4);
}
template <typename CT, int ROWS, int BYTES>
__device__ __forceinline__ void store_staged(const Product& p, uint8_t* own, int64_t row0, int64_t col0, int lane) {
  constexpr int kPer = 16 / (int)sizeof(CT), kChunks = BYTES / 16, kAtOnce = 64 / kChunks;
  __builtin_amdgcn_wave_barrier();
  asm volatile("" ::: "memory");
#pragma unroll
  for (int q = 0; q < ROWS / kAtOnce; ++q) {
    const int r = q * kAtOnce + lane / kChunks, chunk = lane % kChunks;
    float v[kPer];
    load_full<kPer>(reinterpret_cast<const CT*>(staged<BYTES>(own, r, chunk)), v);
    const int64_t row = row0 + r, col = col0 + chunk * kPer, left = p.b.rows - col;
    if (row < p.a.rows && left > 0) {
      const int n = left > kPer ? kPer : (int)left;
      CT* at = reinterpret_cast<CT*>(p.c) + row * p.ldc + col;
      if (p.accumulate) {
        float before[kPer];
        load_some<kPer>(at, n, before);
#pragma unroll
        for (int t = 0; t < kPer; ++t) v[t] += before[t];
      }
      store_some<kPer>(at, n, v);
    }
  }
  __builtin_amdgcn_wave_barrier();
  asm volatile("" ::: "memory");
}

// The results of one row of fragments, 32 x 32 NI: a lane's are sixteen
// consecutive columns of each fragment.  OWN: bytes of the wave's part of LDS.
template <typename CT, int NI, int OWN>
__device__ __forceinline__ void store_wave(const Product& p, uint8_t* own, const v16f (&acc)[NI], int64_t row0, int64_t col0, int lane) {
  constexpr int kPer = 16 / (int)sizeof(CT), kEach = 16 / kPer;  // elements of a chunk; a lane's chunks of a fragment
  constexpr int kTogether = sizeof(CT) == 2 ? NI : 1;            // fragments staged at once
  constexpr int kBytes = kTogether * 32 * (int)sizeof(CT), kRows = OWN / kBytes < 32 ? OWN / kBytes : 32;
  const int fr = lane % 32, fg = lane / 32;
#pragma unroll
  for (int j0 = 0; j0 < NI; j0 += kTogether)
#pragma unroll
    for (int r0 = 0; r0 < 32; r0 += kRows) {
      if (kRows == 32 || fr / kRows == r0 / kRows) {
#pragma unroll
        for (int j = 0; j < kTogether; ++j)
#pragma unroll
          for (int k = 0; k < kEach; ++k) {
            float v[kPer];
#pragma unroll
            for (int t = 0; t < kPer; ++t) v[t] = acc[j0 + j][k * kPer + t];
            store_full<kPer>(reinterpret_cast<CT*>(staged<kBytes>(own, fr % kRows, (j * 2 + fg) * kEach + k)), v);
          }
      }
      store_staged<CT, kRows, kBytes>(p, own, row0 + r0, col0 + j0 * 32, lane);
    }
}

// Item t: a tile and the blocks of its contraction.
struct Item {
  Place at;
  int from, to, split;
};
template <bool PART, int B>
__device__ __forceinline__ Item item_at(const Product& p, int tiles, int t) {
  if (!PART) return {place_of<B, B>(p, t), 0, p.a.blocks, 0};
  const int split = t / tiles, from = split * p.split_blocks;
  return {place_of<B, B>(p, t - split * tiles), from, from + p.split_blocks < p.a.blocks ? from + p.split_blocks : p.a.blocks, split};
}

// Products in tiles of B x B over WR x WC waves, one workgroup per CU that goes
// from item to item: tiles, or with PART the p.splits parts of the contraction
// of each, whose sums go to p.partial.
//
// LDS holds STAGES blocks of each side, loaded straight into it and running on
// into the next item.  (Loads take whole 128-byte lines: of half lines the L2
// gives half as many bytes, 65 GB/s a CU in place of 120.)  A wave reads a
// step's fragments while the matrix cores work on the step before, so it needs
// others only once a block: before the last step, when the block's last
// fragments are in registers, all meet; then its stage is free to be loaded,
// and the next block's is there.  Reads and loads are issued between the matrix
// instructions; a 1 KiB load takes 16 cycles to issue, which holds up a wave's
// matrix instructions where several come together, so with more than two stages
// a block's loads are spread over its halves.
//
// Bound by the matrix cores and the power they draw: 8192^3 with a bf16 c 2.7
// PFLOP/s (the instruction alone, on random data: 4.1; a library's fp8 product
// without block scales 2.7), with an fp32 c 1.45 (1.75 alone).  256 x 256 tiles
// take half the bytes from the L2 per product of 128 x 128 ones; smaller sizes
// lose in their last round of tiles (4096^3 56 and 105 us, 2048^3 12.6 and 24 us).
template <typename CT, bool PART, int B, int WR, int WC, int STAGES, int OWN>
__global__ __launch_bounds__(64 * WR * WC, 1) void k_product8_tiles(Product p) {
  constexpr int kWaves = WR * WC, kMI = B / WR / 32, kNI = B / WC / 32, kLoads = B / (8 * kWaves), kStage = 2 * B * 128;
  constexpr bool kSpread = STAGES > 2;
  using Step = Step8<sizeof(CT) == 4>;
  using Fragment = typename Step::Fragment;
  constexpr int kSteps = Step::kSteps, kCalls = Step::template calls<kMI, kNI>;
  static_assert(kNI == 2 && 128 % (32 * kMI) == 0, "a wave has 64 columns, and its rows share their block of 128 rows");
  static_assert((STAGES * kStage & (STAGES * kStage - 1)) == 0, "the stages' bytes are a power of two");
  extern __shared__ __attribute__((aligned(1024))) uint8_t lds[];
  const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const int tiles = p.tiles_m * p.tiles_n, items = PART ? tiles * p.splits : tiles, per = (items + 7) / 8, xcd = blockIdx.x % 8;
  // this XCD's share of the items, and this workgroup's among them
  const int first = xcd * per + blockIdx.x / 8, past = xcd * per + per < items ? xcd * per + per : items, stride = gridDim.x / 8;
  if (first >= past) return;
  auto item_of = [&](int t) { return item_at<PART, B>(p, tiles, t); };

  // A wave loads eight rows at once: lane l the chunk that belongs at place l
  // % 8 of row l / 8.  Rows go into the lane's offset, which the hardware
  // holds against the matrix's end; the block into the scalar offset.
  const int lr = wave * 8 + lane / 8, lda = (int)p.a.ld, ldb = (int)p.b.ld;
  int va = lr * lda + ((lane % 8) ^ row_key(lr)) * 16, vb = lr * ldb + ((lane % 8) ^ row_key(lr)) * 16;
  // What is loaded next: the item's rows, bytes into them, the last of these, and the stage's place.
  int l_item = first, l_stage = wave * 1024;
  const Item start = item_of(first);
  int l_off = start.from * 128, l_from = l_off, l_end = start.to * 128;
  auto rows_of_a = [&](const Place& at) { return buffer_of(p.a.codes + at.row0 * p.a.ld, (p.a.rows - at.row0) * p.a.ld); };
  auto rows_of_b = [&](const Place& at) { return buffer_of(p.b.codes + at.col0 * p.b.ld, (p.b.rows - at.col0) * p.b.ld); };
  __amdgpu_buffer_rsrc_t ra = rows_of_a(start.at), rb = rows_of_b(start.at);
  auto load_part = [&](int k) {  // 0 .. 2 kLoads - 1: those of a, then those of b
    const bool of_b = k >= kLoads;
    asm("" : "+v"(va), "+v"(vb));  // (offsets of further rows are formed anew: they would each hold a register)
    __builtin_amdgcn_raw_ptr_buffer_load_lds(of_b ? rb : ra, (__attribute__((address_space(3))) void*)(lds + l_stage + k * kWaves * 1024),
                                             16, of_b ? vb + (k - kLoads) * 8 * kWaves * ldb : va + k * 8 * kWaves * lda, l_off, 0, 0);
  };
  auto load_done = [&]() {
    l_stage = (l_stage + kStage) & (STAGES * kStage - 1);
    l_off += 128;
    if (l_off == l_end) {  // past the last item its blocks are loaded again, and not used
      if (l_item + stride < past) {
        l_item += stride;
        const Item it = item_of(l_item);
        l_from = it.from * 128;
        l_end = it.to * 128;
        ra = rows_of_a(it.at);
        rb = rows_of_b(it.at);
      }
      l_off = l_from;
    }
  };

  const int wm = wave / WC * (32 * kMI), wn = wave % WC * 64, fr = lane % 32, fg = lane / 32;
  // Four blocks' scales of each of the lane's rows at once, as the blocks
  // before them end; rows past the end read zeros.
  const int step_a = p.a_scale_shift ? 0 : 32 * 4, step_b = p.b_scale_shift ? 0 : 32 * 4;
  int vsa = ((wm + fr) >> p.a_scale_shift) * 4, vsb = ((wn + row_of_b(fr)) >> p.b_scale_shift) * 4;
  uint32_t ea[kMI], eb[kNI], next_a[kMI], next_b[kNI];
  auto load_scales = [&](const Place& at, int kb) {
    const int64_t r = at.row0 >> p.a_scale_shift, c = at.col0 >> p.b_scale_shift;
    const auto rsa = buffer_of(scale_at(p.a, r, kb & ~3), (p.a.scale_rows - r) * 4);
    const auto rsb = buffer_of(scale_at(p.b, c, kb & ~3), (p.b.scale_rows - c) * 4);
    asm("" : "+v"(vsa), "+v"(vsb));
#pragma unroll
    for (int i = 0; i < kMI; ++i) next_a[i] = (uint32_t)__builtin_amdgcn_raw_buffer_load_b32(rsa, vsa + i * step_a, 0, 0);
#pragma unroll
    for (int j = 0; j < kNI; ++j) next_b[j] = (uint32_t)__builtin_amdgcn_raw_buffer_load_b32(rsb, vsb + j * step_b, 0, 0);
  };
  auto take_scales = [&](int kb) {
#pragma unroll
    for (int i = 0; i < kMI; ++i) ea[i] = next_a[i] >> 8 * (kb & 3);
#pragma unroll
    for (int j = 0; j < kNI; ++j) eb[j] = next_b[j] >> 8 * (kb & 3);
  };

  const int key_a = row_key(fr), key_b = row_key(row_of_b(fr));
  const int a0 = (wm + fr) * 128 + ((2 * fg ^ key_a) << 4), b0 = (B + wn + row_of_b(fr)) * 128 + ((2 * fg ^ key_b) << 4);
  Fragment fa[2][kMI], fb[2][kNI];
  auto read_part = [&](int k, int stage, int half, int step, int to) {  // 0 .. kNI + kMI - 1
    if (k < kNI) fb[to][k] = Step::read(lds + stage, b0 ^ half * 64, k * 4096, step);
    else fa[to][k - kNI] = Step::read(lds + stage, a0 ^ half * 64, (k - kNI) * 4096, step);
  };

  Item item = start;
  load_scales(item.at, item.from);
#pragma unroll
  for (int s = 0; s < STAGES; ++s) {
    // (spread: the last one's second half follows in the first block)
    const int parts = kSpread && s + 1 == STAGES ? kLoads : 2 * kLoads;
#pragma unroll
    for (int k = 0; k < 2 * kLoads; ++k)
      if (k < parts) load_part(k);
    if (parts == 2 * kLoads) load_done();
  }
  take_scales(item.from);
  loads_landed<(STAGES - 1) * 2 * kLoads - (kSpread ? kLoads : 0)>();
  meet();
  int stage = 0;
#pragma unroll
  for (int k = 0; k < kNI + kMI; ++k) read_part(k, 0, 0, 0, 0);
  for (int t = first; t < past; t += stride) {
    const Item next = t + stride < past ? item_of(t + stride) : item;
    v16f acc[kMI][kNI];
#pragma unroll
    for (int i = 0; i < kMI; ++i)
#pragma unroll
      for (int j = 0; j < kNI; ++j)
#pragma unroll
        for (int k = 0; k < 16; ++k) acc[i][j][k] = 0.0f;
    for (int kb = item.from; kb < item.to; ++kb) {
      const bool ends = kb + 1 == item.to, renew = (kb & 3) == 3 || ends;
      if (renew) {
        if (ends) load_scales(next.at, next.from);
        else load_scales(item.at, kb + 1);
      }
      const int after = (stage + kStage) & (STAGES * kStage - 1);
#pragma unroll
      for (int half = 0; half < 2; ++half) {
#pragma unroll
        for (int step = 0; step < kSteps; ++step) {
          const bool ends_half = step + 1 == kSteps, ends_block = ends_half && half == 1;
          const int now = (half * kSteps + step) & 1;
          if (ends_block) {
            reads_landed();
            loads_landed<(STAGES - 2) * 2 * kLoads>();
            meet();
          }
          Step::template multiply<kMI, kNI>(fa[now], fb[now], ea, eb, acc, [&](int c) {
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int k = 0; k < kNI + kMI; ++k)
              if (k * kCalls / (kNI + kMI) == c)
                read_part(k, ends_block ? after : stage, ends_half ? half ^ 1 : half, ends_half ? 0 : step + 1, now ^ 1);
#pragma unroll
            for (int k = 0; k < 2 * kLoads; ++k) {
              if (!kSpread && ends_block && k * kCalls / (2 * kLoads) == c) load_part(k);
              // the first half at the block's end, the second in the next block
              if (kSpread && ends_half && half == (k < kLoads) && (k % kLoads) * kCalls / kLoads == c) load_part(k);
            }
            __builtin_amdgcn_sched_barrier(0);
          });
          if (ends_half && half == (kSpread ? 0 : 1)) load_done();
        }
      }
      stage = after;
      if (renew) {
        take_scales(ends ? next.from : kb + 1);
      } else {
#pragma unroll
        for (int i = 0; i < kMI; ++i) ea[i] >>= 8;
#pragma unroll
        for (int j = 0; j < kNI; ++j) eb[j] >>= 8;
      }
    }
    uint8_t* own = lds + STAGES * kStage + wave * OWN;
    Product to = p;
    if (PART) {
      to.c = p.partial + (int64_t)item.split * p.a.rows * p.b.rows;
      to.ldc = p.b.rows;
      to.accumulate = 0;
    }
#pragma unroll
    for (int i = 0; i < kMI; ++i)
      store_wave<std::conditional_t<PART, float, CT>, kNI, OWN>(to, own, acc[i], item.at.row0 + wm + i * 32, item.at.col0 + wn, lane);
    item = next;
  }
  loads_landed();  // LDS is given back: nothing may still be on its way there
}
constexpr int kBig = 256, kMid = 128;

// c from the parts' sums, added in their order: four columns a thread.
template <typename CT>
__global__ __launch_bounds__(kThreads) void k_product8_join(Product p) {
  const int64_t quads = (p.b.rows + 3) / 4, at = (int64_t)blockIdx.x * kThreads + threadIdx.x, row = at / quads;
  if (row >= p.a.rows) return;
  const int64_t col = (at - row * quads) * 4, plane = p.a.rows * p.b.rows;
  const int n = p.b.rows - col > 4 ? 4 : (int)(p.b.rows - col);
  const float* in = p.partial + row * p.b.rows + col;
  float o[4];
  load_some<4>(in, n, o);
#pragma unroll 4
  for (int k = 1; k < p.splits; ++k) {
    float v[4];
    load_some<4>(in + k * plane, n, v);
#pragma unroll
    for (int t = 0; t < 4; ++t) o[t] += v[t];
  }
  CT* to = reinterpret_cast<CT*>(p.c) + row * p.ldc + col;
  if (p.accumulate) {
    float before[4];
    load_some<4>(to, n, before);
#pragma unroll
    for (int t = 0; t < 4; ++t) o[t] += before[t];
  }
  store_some<4>(to, n, o);
}

// c = 0: a product over no columns, which has no block that the kernels above could
// load.  Four columns a thread, in steps of the grid.  Bound by HBM's writes: 16384 x
// 8192 bf16 43 us, 6.3 TB/s.
template <typename CT>
__global__ __launch_bounds__(kThreads) void k_product8_zero(CT* c, int64_t rows, int64_t cols, int64_t ldc) {
  const int64_t quads = (cols + 3) / 4;
  const float zeros[4] = {0.0f, 0.0f, 0.0f, 0.0f};
  for (int64_t at = (int64_t)blockIdx.x * kThreads + threadIdx.x; at < rows * quads; at += (int64_t)gridDim.x * kThreads) {
    const int64_t row = at / quads, col = (at - row * quads) * 4;
    store_some<4>(c + row * ldc + col, cols - col > 4 ? 4 : (int)(cols - col), zeros);
  }
}

// Products of a few rows (up to 64): what counts is to read b once, with as
// many loads in flight as the chip takes.  A workgroup has sixteen or 32 rows
// of b (columns of c), whose blocks its waves take in turn, straight from memory
// into registers; their sums meet in LDS, in the order of the waves.  XT
// uint8_t: a is given as 8-bit blocks; else as it is, up to sixteen rows of
// it, which every workgroup quantizes as it reads them (one launch less).
// Bound by latency, then by HBM: 8 x 8192 x 2048 (17 MB) 5.8 us, 64 rows 9.3 us,
// 1 x 8192 x 8192 (67 MB) 14.4 us, 4.7 TB/s.
struct Few {
  const void* x;
  int64_t ldx, m, k;
  Mat a;  // a's blocks, or nothing
  int32_t a_scale_shift;
  Mat b;
  int32_t b_scale_shift, accumulate;
  void* c;
  int64_t ldc;
};

// NJ: sixteens of columns of a workgroup; kAtOnce: blocks that a wave has in flight
// (more of them do not fit the registers).
template <typename XT, typename CT, int MI, int NJ, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void k_product8_few(Few p) {
  constexpr bool kCodes = sizeof(XT) == 1;
  constexpr int kAtOnce = sizeof(XT) == 4 || MI > 1 || (sizeof(XT) == 2 && WAVES > 8) ? 2 : 4;
  static_assert(kCodes || MI == 1, "sixteen rows");
  using Rows = Raw<std::conditional_t<kCodes, bf16_t, XT>>;
  __shared__ v4f part[WAVES][MI * NJ][64];
  const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), r = lane % 16, g = lane / 16;
  const int64_t col0 = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * (16 * NJ);
  const uint8_t* b[NJ];
  int64_t bs[NJ];
#pragma unroll
  for (int j = 0; j < NJ; ++j) {
    const int64_t br = col0 + j * 16 + r < p.b.rows ? col0 + j * 16 + r : p.b.rows - 1;
    b[j] = p.b.codes + br * p.b.ld + g * 32;
    bs[j] = br >> p.b_scale_shift;
  }
  const XT* a[MI];
  int64_t as[MI];
#pragma unroll
  for (int i = 0; i < MI; ++i) {
    const int64_t ar = i * 16 + r < p.m ? i * 16 + r : p.m - 1;
    a[i] = reinterpret_cast<const XT*>(p.x) + ar * p.ldx + g * 32;
    as[i] = ar >> p.a_scale_shift;
  }
  v4f acc[MI][NJ];
#pragma unroll
  for (int i = 0; i < MI; ++i)
#pragma unroll
    for (int j = 0; j < NJ; ++j) acc[i][j] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
  for (int k0 = wave; k0 < p.b.blocks; k0 += kAtOnce * WAVES) {
    v8i fb[kAtOnce][NJ], fa[kAtOnce][MI];
    uint32_t eb[kAtOnce][NJ], ea[kAtOnce][MI];
    Rows raw[kCodes ? 1 : kAtOnce][4];
#pragma unroll
    for (int u = 0; u < kAtOnce; ++u) {
      const int kb = k0 + u * WAVES, e = kb * kBlock8;
      if (kb >= p.b.blocks) break;
#pragma unroll
      for (int j = 0; j < NJ; ++j) {
        const v4i lo = *reinterpret_cast<const v4i*>(b[j] + e), hi = *reinterpret_cast<const v4i*>(b[j] + e + 16);
        fb[u][j] = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
        eb[u][j] = *scale_at(p.b, bs[j], kb);
      }
      if constexpr (kCodes) {
#pragma unroll
        for (int i = 0; i < MI; ++i) {
          const v4i lo = *reinterpret_cast<const v4i*>(a[i] + e), hi = *reinterpret_cast<const v4i*>(a[i] + e + 16);
          fa[u][i] = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
          ea[u][i] = *scale_at(p.a, as[i], kb);
        }
      } else {
#pragma unroll
        for (int v = 0; v < 4; ++v) raw[u][v].load(a[0] + e + v * kE, (int)(p.k - e) - g * 32 - v * kE);
      }
    }
#pragma unroll
    for (int u = 0; u < kAtOnce; ++u) {
      if (k0 + u * WAVES >= p.b.blocks) break;
      if constexpr (!kCodes) {
        float x[4][kE], most = 0.0f;
#pragma unroll
        for (int v = 0; v < 4; ++v) {
          raw[u][v].values(x[v]);
#pragma unroll
          for (int t = 0; t < kE; ++t) most = max_abs(most, x[v][t]);
        }
        if (is_infinite(most)) {
          most = 0.0f;
#pragma unroll
          for (int v = 0; v < 4; ++v)
#pragma unroll
            for (int t = 0; t < kE; ++t) most = fmaxf(most, finite_abs(x[v][t]));
        }
        ea[u][0] = scale_byte(max_with32(max_with16(most)));
        const float inv = inverse_scale_of(ea[u][0]);
#pragma unroll
        for (int v = 0; v < 4; ++v) {
          fa[u][0][2 * v] = (int)codes_of(x[v][0] * inv, x[v][1] * inv, x[v][2] * inv, x[v][3] * inv);
          fa[u][0][2 * v + 1] = (int)codes_of(x[v][4] * inv, x[v][5] * inv, x[v][6] * inv, x[v][7] * inv);
        }
      }
      if constexpr (sizeof(CT) == 2) {
#pragma unroll
        for (int i = 0; i < MI; ++i)
#pragma unroll
          for (int j = 0; j < NJ; ++j)
            acc[i][j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(fb[u][j], fa[u][i], acc[i][j], 0, 0, 0, eb[u][j], 0, ea[u][i]);
      } else {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          v8bf wb[NJ];
#pragma unroll
          for (int j = 0; j < NJ; ++j) wb[j] = widened(fb[u][j][2 * k], fb[u][j][2 * k + 1], scale_of(eb[u][j]));
#pragma unroll
          for (int i = 0; i < MI; ++i) {
            const v8bf wa = widened(fa[u][i][2 * k], fa[u][i][2 * k + 1], scale_of(ea[u][i]));
#pragma unroll
            for (int j = 0; j < NJ; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wb[j], wa, acc[i][j], 0, 0, 0);
          }
        }
      }
    }
  }
#pragma unroll
  for (int i = 0; i < MI; ++i)
#pragma unroll
    for (int j = 0; j < NJ; ++j) part[wave][i * NJ + j][lane] = acc[i][j];
  __syncthreads();
  for (int f = wave; f < MI * NJ; f += WAVES) {
    v4f s = part[0][f][lane];
#pragma unroll
    for (int w = 1; w < WAVES; ++w) s += part[w][f][lane];
    const int64_t row = f / NJ * 16 + r, col = col0 + f % NJ * 16 + g * 4, left = p.b.rows - col;
    if (row < p.m && left > 0) {
      const int n = left > 4 ? 4 : (int)left;
      CT* at = reinterpret_cast<CT*>(p.c) + row * p.ldc + col;
      float o[4] = {s[0], s[1], s[2], s[3]};
      if (p.accumulate) {
        float before[4];
        load_some<4>(at, n, before);
#pragma unroll
        for (int t = 0; t < 4; ++t) o[t] += before[t];
      }
      store_some<4>(at, n, o);
    }
  }
}

// --------------------------------------------------------------------- host

template <int V>
using Int = std::integral_constant<int, V>;

int64_t up(int64_t n, int64_t m) { return (n + m - 1) / m * m; }

constexpr int64_t kMostCols = INT64_C(1) << 22;  // a tile's rows stay within 2^31 bytes

// How a product of m x n x k goes over the chip.  Up to 64 rows the kernel for
// few rows, with more than sixteen while the contraction is short: a workgroup
// takes all of it (64 x 4096 x 4096 12.9 us, in parts of tiles 14.3 us; 64 x
// 2048 x 8192 26.8 us, in parts 15.9 us; 24 x 2048 x 8192 13.4 us, in parts
// 12.6 us).  Tiles of 256 x 256 from two tiles of 128 x 128 a CU on, unless
// that pads more than a quarter (2000 x 4000 x 1024, 512 such tiles: 17.5 us
// in 128 large ones, 14.4 us).  Else tiles of 128 x 128: with more than one a
// CU two workgroups a CU of two stages each (`shared`; 1999 x 2304 x 768 12.1
// us one after the other, 10.5 us); where they leave CUs idle, the contraction
// in parts of at least four blocks (1536 x 512 x 8191 45 us whole, 19 us).
constexpr int64_t kFew = 64, kFewWhole = 16;  // rows; of which quantized on the way
struct Shape {
  bool few, big, shared;
  int32_t splits, split_blocks;
};
Shape shape_of(int64_t m, int64_t n, int64_t k) {
  const int64_t blocks = up(k, kBlock8) / kBlock8;
  const bool few = m <= 16 || (m <= kFew && (m <= 32 ? 2 : 4) * blocks <= 128);
  Shape s = {few, false, false, 1, (int32_t)blocks};
  if (s.few) return s;
  const int64_t big = (up(m, kBig) / kBig) * (up(n, kBig) / kBig), tiles = (up(m, kMid) / kMid) * (up(n, kMid) / kMid);
  s.big = tiles > 512 && 4 * big <= tiles + tiles / 4;
  s.shared = !s.big && tiles > 256;
  if (!s.big && tiles > 0 && tiles <= 128 && blocks >= 8) {
    const int64_t parts = std::min<int64_t>(256 / tiles, blocks / 4);
    s.split_blocks = (int32_t)((blocks + parts - 1) / parts);
    s.splits = (int32_t)((blocks + s.split_blocks - 1) / s.split_blocks);
  }
  return s;
}
size_t product_bytes(int64_t m, int64_t n, int64_t k) {
  const Shape s = shape_of(m, n, k);
  return s.splits > 1 ? (size_t)s.splits * (size_t)m * (size_t)n * sizeof(float) : 0;
}

int32_t check_matrix(const mtdao_matrix8& q, const char* name, std::string* e) {
  if (q.rows < 0 || q.cols < 0) return fail(e, MTDAO_ERR_INVALID_ARG, "%s: rows or cols < 0", name);
  if (q.cols > kMostCols) return fail(e, MTDAO_ERR_INVALID_ARG, "%s: cols exceed 2^22", name);
  if (q.rows > INT64_C(0x7fffffff)) return fail(e, MTDAO_ERR_INVALID_ARG, "%s: rows exceed 2^31", name);
  if (q.ld % kBlock8 != 0 || q.ld < q.cols || q.ld > 2 * kMostCols)
    return fail(e, MTDAO_ERR_INVALID_ARG, "%s: ld is not a multiple of 128 from cols on", name);
  if (q.scale_rows != 1 && q.scale_rows != kBlock8)
    return fail(e, MTDAO_ERR_INVALID_ARG, "%s: scale_rows is not 1 or 128", name);
  if (q.scale_ld != 4 * ((q.rows + q.scale_rows - 1) / q.scale_rows))
    return fail(e, MTDAO_ERR_INVALID_ARG, "%s: scale_ld is not 4 ceil(rows / scale_rows)", name);
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
  m.scale_rows = (q->rows + q->scale_rows - 1) / q->scale_rows;
  m.ld = q->ld;
  m.blocks = (int32_t)(up(q->cols, kBlock8) / kBlock8);
  m.scale_ld = q->scale_ld;
  return m;
}

int64_t scale_bytes(const mtdao_matrix8& q) { return up(q.cols, 4 * kBlock8) / (4 * kBlock8) * q.scale_ld; }
int64_t esize(int32_t dt) { return dt == MTDAO_BF16 ? 2 : 4; }

// A [rows][cols] input with row stride ld.
int32_t check_input(const void* x, int32_t dtype, int64_t rows, int64_t cols, int64_t ld, const char* name, std::string* e) {
  if (dtype != MTDAO_F32 && dtype != MTDAO_BF16) return fail(e, MTDAO_ERR_INVALID_ARG, "dtype must be F32(0) or BF16(1)");
  if (rows == 0 || cols == 0) return MTDAO_OK;
  if (ld < cols || ld > (INT64_C(1) << 40) / rows)
    return fail(e, MTDAO_ERR_INVALID_ARG, "row stride %lld of %s is below its columns or exceeds 2^40 elements in all", (long long)ld, name);
  if (!x) return fail(e, MTDAO_ERR_INVALID_ARG, "%s is NULL", name);
  if (!aligned_to(x, (uintptr_t)esize(dtype))) return fail(e, MTDAO_ERR_ALIGN, "%s is not aligned to its element", name);
  return MTDAO_OK;
}

int32_t check_product(const mtdao_matrix8& a, const mtdao_matrix8& b, const void* c, int32_t c_dtype, int64_t ldc,
                      int32_t accumulate, std::string* e) {
  if (a.cols != b.cols) return fail(e, MTDAO_ERR_INVALID_ARG, "a has %lld columns, b has %lld", (long long)a.cols, (long long)b.cols);
  if (c_dtype != MTDAO_F32 && c_dtype != MTDAO_BF16) return fail(e, MTDAO_ERR_INVALID_ARG, "c_dtype must be F32(0) or BF16(1)");
  if (accumulate && c_dtype != MTDAO_F32) return fail(e, MTDAO_ERR_INVALID_ARG, "accumulate needs an fp32 c");
  if (a.rows == 0 || b.rows == 0) return MTDAO_OK;
  if (ldc < b.rows || ldc > (INT64_C(1) << 40) / a.rows)
    return fail(e, MTDAO_ERR_INVALID_ARG, "ldc %lld is below the columns of c or exceeds 2^40 elements in all", (long long)ldc);
  if (!c) return fail(e, MTDAO_ERR_INVALID_ARG, "c is NULL");
  if (!aligned_to(c, (uintptr_t)esize(c_dtype))) return fail(e, MTDAO_ERR_ALIGN, "c is not aligned to its element");
  const int64_t cbytes = ((a.rows - 1) * ldc + b.rows) * esize(c_dtype);
  for (const mtdao_matrix8* m : {&a, &b})
    if (overlap(c, cbytes, m->codes, m->rows * m->ld) || overlap(c, cbytes, m->scales, scale_bytes(*m)))
      return fail(e, MTDAO_ERR_INVALID_ARG, "c overlaps a or b");
  return MTDAO_OK;
}

int32_t check_workspace(const void* workspace, size_t given, size_t need, std::string* e) {
  if (need == 0) return MTDAO_OK;
  if (!workspace || given < need)
    return fail(e, MTDAO_ERR_WORKSPACE, "workspace of %zu bytes required, %zu given", need, workspace ? given : (size_t)0);
  if (!aligned_to(workspace, 256)) return fail(e, MTDAO_ERR_ALIGN, "workspace is not 256-byte aligned");
  return MTDAO_OK;
}

Quantized quantized_of(const void* x, int64_t ld, const mtdao_matrix8* q, const mtdao_matrix8* qt) {
  const int64_t cols = q ? q->cols : qt->rows;
  return {x, ld, cols, mat_of(q), mat_of(qt), (int32_t)(up(cols, kBlock8) / kBlock8)};
}

// Tiles of one matrix, or of two (`two.tiles` not 0) of as many rows.
int32_t launch_tiles(const Quantized& one, const Quantized& two, int32_t dtype, int64_t rows, bool square, hipStream_t st, std::string* e) {
  const int64_t ty = up(rows, kBlock8) / kBlock8;
  if (ty > 65535 || (int64_t)one.tiles + two.tiles > 0x7fffff) return fail(e, MTDAO_ERR_INVALID_ARG, "the matrix exceeds the largest launch");
  const dim3 grid((unsigned)(one.tiles + two.tiles), (unsigned)ty), block(kTileThreads);
  auto with = [&](auto t) {
    using T = decltype(t);
    if (square) hipLaunchKernelGGL((k_quantize8_tile<T, true>), grid, block, 0, st, one, two, rows);
    else hipLaunchKernelGGL((k_quantize8_tile<T, false>), grid, block, 0, st, one, two, rows);
  };
  if (dtype == MTDAO_BF16) with(bf16_t{});
  else with(float{});
  return MTDAO_OK;
}

int32_t launch_quantize(const void* x, int32_t dtype, int64_t ld, const mtdao_matrix8* q, const mtdao_matrix8* qt, hipStream_t st,
                        std::string* e) {
  const int64_t rows = q ? q->rows : qt->cols, cols = q ? q->cols : qt->rows;
  const bool square = (q ? q : qt)->scale_rows == kBlock8;
  if (qt || square) return launch_tiles(quantized_of(x, ld, q, qt), Quantized{}, dtype, rows, square, st, e);
  const Mat m = mat_of(q);
  const int groups = (m.blocks + 3) / 4;
  const int64_t all = (rows + 3) / 4, fours = std::min(all, INT64_C(0xffffff) / groups);  // fewer than 2^32 threads along x
  const int64_t along_y = (all + fours - 1) / fours;
  if (along_y > 65535) return fail(e, MTDAO_ERR_INVALID_ARG, "the matrix exceeds the largest launch");
  const dim3 grid((unsigned)(fours * groups), (unsigned)along_y), block(kThreads);
  if (dtype == MTDAO_BF16) hipLaunchKernelGGL(k_quantize8_rows<bf16_t>, grid, block, 0, st, static_cast<const bf16_t*>(x), ld, cols, groups, (int)fours, m);
  else hipLaunchKernelGGL(k_quantize8_rows<float>, grid, block, 0, st, static_cast<const float*>(x), ld, cols, groups, (int)fours, m);
  return MTDAO_OK;
}

// Waves of a workgroup of the kernel for few rows: enough that each has a few
// blocks.  Its columns: sixteen, or 32 where a's blocks, read by every workgroup, are
// much (from 17 rows on) and sixteen would take more than one workgroup a CU, 4096
// columns (with 32 against sixteen: 64 x 4096 x 2048 8.6 us (7.4), 64 x 5120 x 2048 8.6
// us (13.0), 64 x 8192 x 2048 8.7 us (13.1); 24 x 4096 x 768 3.8 us (3.3), 24 x 5120 x 768
// 3.8 us (4.1), 24 x 8192 x 8192 18.0 us (25.1); between 24 and 64 rows and 256 and 8192
// columns of a the turn is at 4096 everywhere, for either c).
constexpr int64_t kWideFrom = 4096;
template <typename XT, typename CT, int MI>
void launch_few(const Few& f, hipStream_t st) {
  auto go = [&](auto nj, auto waves) {
    constexpr int NJ = decltype(nj)::value, W = decltype(waves)::value;
    hipLaunchKernelGGL((k_product8_few<XT, CT, MI, NJ, W>), grid_of((f.b.rows + 16 * NJ - 1) / (16 * NJ)), dim3(64 * W), 0, st, f);
  };
  if constexpr (MI > 1) {
    if (f.b.rows > kWideFrom) return go(Int<2>{}, Int<8>{});
  }
  if constexpr (MI < 4) {  // (four fragments of rows: at most 32 blocks)
    if (f.b.blocks > 32) return go(Int<1>{}, Int<16>{});
  }
  go(Int<1>{}, Int<8>{});
}

Few few_of(const mtdao_matrix8& b, void* c, int64_t ldc, int32_t accumulate, int64_t m) {
  Few f = {};
  f.b = mat_of(&b);
  f.b_scale_shift = b.scale_rows == 1 ? 0 : 7;
  f.c = c;
  f.ldc = ldc;
  f.accumulate = accumulate;
  f.m = m;
  f.k = b.cols;
  return f;
}

int32_t launch_few_whole(const void* x, int32_t dtype, int64_t rows, int64_t ld, const mtdao_matrix8& w, void* y, int32_t y_dtype,
                         int64_t ldy, hipStream_t st) {
  Few f = few_of(w, y, ldy, 0, rows);
  f.x = x;
  f.ldx = ld;
  if (dtype == MTDAO_BF16 && y_dtype == MTDAO_BF16) launch_few<bf16_t, bf16_t, 1>(f, st);
  else if (dtype == MTDAO_BF16) launch_few<bf16_t, float, 1>(f, st);
  else if (y_dtype == MTDAO_BF16) launch_few<float, bf16_t, 1>(f, st);
  else launch_few<float, float, 1>(f, st);
  return MTDAO_OK;
}

// More than 64 KiB of LDS for a kernel, asked for once per kernel and device.
int32_t allow_lds(const void* kernel, int bytes, std::string* e) try {
  static std::mutex lock;
  static std::set<std::pair<const void*, int>> done;
  int device = 0;
  int32_t r = hip_check(e, hipGetDevice(&device), "mtdao_product8 device");
  if (r != MTDAO_OK) return r;
  std::lock_guard<std::mutex> held(lock);
  if (done.count({kernel, device})) return MTDAO_OK;
  r = hip_check(e, hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, bytes), "mtdao_product8 LDS");
  if (r == MTDAO_OK) done.insert({kernel, device});
  return r;
} catch (const std::bad_alloc&) {
  return fail(e, MTDAO_ERR_WORKSPACE, "out of host memory");
}

// a, b, c: checked; c has elements.
int32_t launch_product(const mtdao_matrix8& a, const mtdao_matrix8& b, void* c, int32_t c_dtype, int64_t ldc, int32_t accumulate,
                       void* workspace, hipStream_t st, std::string* e) {
  if (a.cols == 0) {  // no codes, no scales: their addresses may be anything
    if (accumulate) return MTDAO_OK;
    const int64_t quads = a.rows * ((b.rows + 3) / 4);
    const dim3 grid((unsigned)std::min<int64_t>((quads + kThreads - 1) / kThreads, 4096)), block(kThreads);
    auto zero = [&](auto ct) {
      using CT = decltype(ct);
      hipLaunchKernelGGL(k_product8_zero<CT>, grid, block, 0, st, static_cast<CT*>(c), a.rows, b.rows, ldc);
    };
    if (c_dtype == MTDAO_F32) zero(float{});
    else zero(bf16_t{});
    return MTDAO_OK;
  }
  const Shape shape = shape_of(a.rows, b.rows, a.cols);
  if (shape.few) {
    Few f = few_of(b, c, ldc, accumulate, a.rows);
    f.x = a.codes;
    f.ldx = a.ld;
    f.a = mat_of(&a);
    f.a_scale_shift = a.scale_rows == 1 ? 0 : 7;
    auto with = [&](auto ct) {
      using CT = decltype(ct);
      if (a.rows <= 16) launch_few<uint8_t, CT, 1>(f, st);
      else if (a.rows <= 32) launch_few<uint8_t, CT, 2>(f, st);
      else launch_few<uint8_t, CT, 4>(f, st);
    };
    if (c_dtype == MTDAO_F32) with(float{});
    else with(bf16_t{});
    return MTDAO_OK;
  }
  Product p = {};
  p.a = mat_of(&a);
  p.b = mat_of(&b);
  p.c = c;
  p.ldc = ldc;
  p.a_scale_shift = a.scale_rows == 1 ? 0 : 7;
  p.b_scale_shift = b.scale_rows == 1 ? 0 : 7;
  p.accumulate = accumulate;
  p.group = 8;
  p.splits = shape.splits;
  p.split_blocks = shape.split_blocks;
  p.partial = static_cast<float*>(workspace);
  // own: LDS of a wave for its results; each: workgroups of a CU
  auto go = [&](auto kernel, int tile, int stages, int own, int each) {
    p.tiles_m = (int32_t)(up(a.rows, tile) / tile);
    p.tiles_n = (int32_t)(up(b.rows, tile) / tile);
    const int64_t items = (int64_t)p.tiles_m * p.tiles_n * p.splits;
    if (items > INT64_C(0x3fffffff)) return fail(e, MTDAO_ERR_INVALID_ARG, "c has more tiles than one launch takes");
    const int bytes = stages * 2 * tile * 128 + 8 * own;
    const int32_t r = allow_lds(reinterpret_cast<const void*>(kernel), bytes, e);
    if (r != MTDAO_OK) return r;
    hipLaunchKernelGGL(kernel, dim3((unsigned)std::min<int64_t>(up(items, 8), 256 * each)), dim3(512), bytes, st, p);
    return (int32_t)MTDAO_OK;
  };
  auto pick = [&](auto ct) {
    using CT = decltype(ct);
    if (shape.big) return go(k_product8_tiles<CT, false, kBig, 2, 4, 2, 4096>, kBig, 2, 4096, 1);
    if (shape.shared) return go(k_product8_tiles<CT, false, kMid, 4, 2, 2, 2048>, kMid, 2, 2048, 2);
    if (shape.splits == 1) return go(k_product8_tiles<CT, false, kMid, 4, 2, 4, 4096>, kMid, 4, 4096, 1);
    const int32_t done = go(k_product8_tiles<CT, true, kMid, 4, 2, 4, 4096>, kMid, 4, 4096, 1);
    if (done != MTDAO_OK) return done;
    const int64_t quads = p.a.rows * ((p.b.rows + 3) / 4);
    hipLaunchKernelGGL(k_product8_join<CT>, dim3((unsigned)((quads + kThreads - 1) / kThreads)), dim3(kThreads), 0, st, p);
    return done;
  };
  return c_dtype == MTDAO_F32 ? pick(float{}) : pick(bf16_t{});
}

// Where a linear layer's 8-bit matrices and partial sums are in its workspace.
int64_t up256(int64_t n) { return up(n, 256); }
struct Part {
  int64_t codes, scales, end;
};
// An odd number of blocks from row to row: in rows a multiple of 2 KiB apart the
// lines that a tile takes at once lie in few of the L2's channels (2048 x 2048
// x 8192 40.2 us so, x 8320 35.7 us).
int64_t spread_ld(int64_t cols) {
  const int64_t blocks = up(cols, kBlock8) / kBlock8;
  return (blocks | 1) * kBlock8;
}
Part part_at(int64_t at, int64_t rows, int64_t cols) {
  const int64_t scales = at + up256(rows * spread_ld(cols));
  return {at, scales, scales + up256(up(cols, 4 * kBlock8) / (4 * kBlock8) * 4 * rows)};
}
mtdao_matrix8 matrix_at(void* workspace, int64_t codes, int64_t scales, int64_t rows, int64_t cols) {
  mtdao_matrix8 m = {};
  m.codes = static_cast<uint8_t*>(workspace) + codes;
  m.scales = static_cast<uint8_t*>(workspace) + scales;
  m.rows = rows;
  m.cols = cols;
  m.ld = spread_ld(cols);
  m.scale_ld = 4 * rows;
  m.scale_rows = 1;
  return m;
}
struct Forward {
  int64_t codes, scales, product;
  size_t bytes;
};
Forward forward_layout(int64_t m, int64_t n, int64_t k) {
  if (m <= kFewWhole || n == 0 || k == 0) return {0, 0, 0, 0};
  const Part q = part_at(0, m, k);
  return {q.codes, q.scales, q.end, (size_t)q.end + product_bytes(m, n, k)};
}
struct Backward {
  Part dy, dyt, xt;
  int64_t product;
  size_t bytes;
};
Backward backward_layout(int64_t m, int64_t n, int64_t k) {
  Backward b = {};
  b.dy = part_at(0, m, n);
  b.dyt = part_at(b.dy.end, n, m);
  b.xt = part_at(b.dyt.end, k, m);
  b.product = b.xt.end;
  b.bytes = (size_t)b.product + std::max(product_bytes(m, k, n), product_bytes(n, k, m));
  return b;
}

}  // namespace

extern "C" {

int32_t mtdao_quantize8(const void* x, int32_t dtype, int64_t ld, const mtdao_matrix8* q, const mtdao_matrix8* qt,
                        void* hip_stream) {
  std::string* e = &g_err;
  if (!q && !qt) return fail(e, MTDAO_ERR_INVALID_ARG, "q and qt are NULL");
  int32_t r = MTDAO_OK;
  if (q) r = check_matrix(*q, "q", e);
  if (r == MTDAO_OK && qt) r = check_matrix(*qt, "qt", e);
  if (r != MTDAO_OK) return r;
  if (q && qt && (q->rows != qt->cols || q->cols != qt->rows || q->scale_rows != qt->scale_rows))
    return fail(e, MTDAO_ERR_INVALID_ARG, "qt is not q transposed");
  const int64_t rows = q ? q->rows : qt->cols, cols = q ? q->cols : qt->rows;
  r = check_input(x, dtype, rows, cols, ld, "x", e);
  if (r != MTDAO_OK || rows == 0 || cols == 0) return r;
  const int64_t xbytes = ((rows - 1) * ld + cols) * esize(dtype);
  for (const mtdao_matrix8* o : {q, qt})
    if (o && (overlap(x, xbytes, o->codes, o->rows * o->ld) || overlap(x, xbytes, o->scales, scale_bytes(*o))))
      return fail(e, MTDAO_ERR_INVALID_ARG, "x overlaps an output");
  RoctxRange range("mtdao_quantize8 rows=%lld cols=%lld", (long long)rows, (long long)cols);
  r = launch_quantize(x, dtype, ld, q, qt, reinterpret_cast<hipStream_t>(hip_stream), e);
  return r != MTDAO_OK ? r : hip_check(e, hipGetLastError(), "mtdao_quantize8 launch");
}

int32_t mtdao_product8_workspace_bytes(int64_t m, int64_t n, int64_t k, size_t* bytes) {
  if (!bytes) return fail(&g_err, MTDAO_ERR_INVALID_ARG, "bytes is NULL");
  if (m < 0 || n < 0 || k < 0) return fail(&g_err, MTDAO_ERR_INVALID_ARG, "a size is below 0");
  if (m > INT64_C(0x7fffffff) || n > INT64_C(0x7fffffff) || k > kMostCols)
    return fail(&g_err, MTDAO_ERR_INVALID_ARG, "a size exceeds what mtdao_product8 takes");
  *bytes = product_bytes(m, n, k);
  return MTDAO_OK;
}

int32_t mtdao_product8(const mtdao_matrix8* a, const mtdao_matrix8* b, void* c, int32_t c_dtype, int64_t ldc,
                       int32_t accumulate, void* workspace, size_t workspace_bytes, void* hip_stream) {
  std::string* e = &g_err;
  if (!a || !b) return fail(e, MTDAO_ERR_INVALID_ARG, "a or b is NULL");
  int32_t r = check_matrix(*a, "a", e);
  if (r == MTDAO_OK) r = check_matrix(*b, "b", e);
  if (r == MTDAO_OK) r = check_product(*a, *b, c, c_dtype, ldc, accumulate, e);
  if (r != MTDAO_OK) return r;
  if (a->rows == 0 || b->rows == 0) return MTDAO_OK;
  r = check_workspace(workspace, workspace_bytes, product_bytes(a->rows, b->rows, a->cols), e);
  if (r != MTDAO_OK) return r;
  RoctxRange range("mtdao_product8 m=%lld n=%lld k=%lld", (long long)a->rows, (long long)b->rows, (long long)a->cols);
  r = launch_product(*a, *b, c, c_dtype, ldc, accumulate, workspace, reinterpret_cast<hipStream_t>(hip_stream), e);
  return r != MTDAO_OK ? r : hip_check(e, hipGetLastError(), "mtdao_product8 launch");
}

int32_t mtdao_linear8_workspace_bytes(int64_t m, int64_t n, int64_t k, size_t* forward, size_t* backward) {
  if (!forward || !backward) return fail(&g_err, MTDAO_ERR_INVALID_ARG, "forward or backward is NULL");
  if (m < 0 || n < 0 || k < 0 || m > kMostCols || n > kMostCols || k > kMostCols)
    return fail(&g_err, MTDAO_ERR_INVALID_ARG, "a size is below 0 or above 2^22");
  *forward = forward_layout(m, n, k).bytes;
  *backward = backward_layout(m, n, k).bytes;
  return MTDAO_OK;
}

int32_t mtdao_linear8(const void* x, int32_t dtype, int64_t rows, int64_t ld, const mtdao_matrix8* w, void* y, int32_t y_dtype,
                      int64_t ldy, void* workspace, size_t workspace_bytes, void* hip_stream) {
  std::string* e = &g_err;
  if (!w) return fail(e, MTDAO_ERR_INVALID_ARG, "w is NULL");
  int32_t r = check_matrix(*w, "w", e);
  if (r == MTDAO_OK && (rows < 0 || rows > kMostCols)) r = fail(e, MTDAO_ERR_INVALID_ARG, "rows below 0 or above 2^22");
  if (r == MTDAO_OK) r = check_input(x, dtype, rows, w->cols, ld, "x", e);
  if (r != MTDAO_OK) return r;
  const Forward f = forward_layout(rows, w->rows, w->cols);
  mtdao_matrix8 q = matrix_at(workspace, f.codes, f.scales, rows, w->cols);
  r = check_product(q, *w, y, y_dtype, ldy, 0, e);
  if (r == MTDAO_OK && rows > 0 && w->rows > 0) {
    r = check_workspace(workspace, workspace_bytes, f.bytes, e);
    if (r == MTDAO_OK && overlap(y, ((rows - 1) * ldy + w->rows) * esize(y_dtype), x, ((rows - 1) * ld + w->cols) * esize(dtype)))
      r = fail(e, MTDAO_ERR_INVALID_ARG, "y overlaps x");
  }
  if (r != MTDAO_OK || rows == 0 || w->rows == 0) return r;
  hipStream_t st = reinterpret_cast<hipStream_t>(hip_stream);
  RoctxRange range("mtdao_linear8 m=%lld n=%lld k=%lld", (long long)rows, (long long)w->rows, (long long)w->cols);
  if (rows <= kFewWhole && w->cols > 0) {
    r = launch_few_whole(x, dtype, rows, ld, *w, y, y_dtype, ldy, st);
  } else {
    if (w->cols > 0) r = launch_quantize(x, dtype, ld, &q, nullptr, st, e);
    if (r == MTDAO_OK)
      r = launch_product(q, *w, y, y_dtype, ldy, 0, static_cast<char*>(workspace) + f.product, st, e);
  }
  return r != MTDAO_OK ? r : hip_check(e, hipGetLastError(), "mtdao_linear8 launch");
}

int32_t mtdao_linear8_backward(const void* dy, const void* x, int32_t dtype, int64_t rows, int64_t ld_dy, int64_t ld_x,
                               const mtdao_matrix8* wt, void* dx, int64_t ld_dx, float* dw, int64_t ld_dw, int32_t accumulate,
                               void* workspace, size_t workspace_bytes, void* hip_stream) {
  std::string* e = &g_err;
  if (!wt) return fail(e, MTDAO_ERR_INVALID_ARG, "wt is NULL");
  int32_t r = check_matrix(*wt, "wt", e);
  if (r == MTDAO_OK && (rows < 0 || rows > kMostCols)) r = fail(e, MTDAO_ERR_INVALID_ARG, "rows below 0 or above 2^22");
  const int64_t n = wt->cols, k = wt->rows;
  if (r == MTDAO_OK) r = check_input(dy, dtype, rows, n, ld_dy, "dy", e);
  if (r == MTDAO_OK) r = check_input(x, dtype, rows, k, ld_x, "x", e);
  if (r != MTDAO_OK) return r;
  const Backward f = backward_layout(rows, n, k);
  mtdao_matrix8 q = matrix_at(workspace, f.dy.codes, f.dy.scales, rows, n);
  mtdao_matrix8 qt = matrix_at(workspace, f.dyt.codes, f.dyt.scales, n, rows);
  mtdao_matrix8 xt = matrix_at(workspace, f.xt.codes, f.xt.scales, k, rows);
  r = check_product(q, *wt, dx, dtype, ld_dx, 0, e);
  if (r == MTDAO_OK) r = check_product(qt, xt, dw, MTDAO_F32, ld_dw, accumulate, e);
  if (r == MTDAO_OK && n > 0 && k > 0) r = check_workspace(workspace, workspace_bytes, f.bytes, e);
  if (r == MTDAO_OK && rows > 0 && n > 0 && k > 0) {
    const int64_t es = esize(dtype);
    const struct { const void* p; int64_t bytes; } out[2] = {{dx, ((rows - 1) * ld_dx + k) * es}, {dw, ((n - 1) * ld_dw + k) * 4}},
                                                   in[2] = {{dy, ((rows - 1) * ld_dy + n) * es}, {x, ((rows - 1) * ld_x + k) * es}};
    for (auto& o : out)
      for (auto& i : in)
        if (overlap(o.p, o.bytes, i.p, i.bytes)) return fail(e, MTDAO_ERR_INVALID_ARG, "dx or dw overlaps dy or x");
    if (overlap(out[0].p, out[0].bytes, out[1].p, out[1].bytes)) return fail(e, MTDAO_ERR_INVALID_ARG, "dx overlaps dw");
    if (overlap(dw, out[1].bytes, wt->codes, wt->rows * wt->ld) || overlap(dw, out[1].bytes, wt->scales, scale_bytes(*wt)))
      return fail(e, MTDAO_ERR_INVALID_ARG, "dw overlaps wt");
  }
  if (r != MTDAO_OK) return r;
  hipStream_t st = reinterpret_cast<hipStream_t>(hip_stream);
  RoctxRange range("mtdao_linear8_backward m=%lld n=%lld k=%lld", (long long)rows, (long long)n, (long long)k);
  if (rows > 0 && n > 0 && k > 0) {
    r = launch_tiles(quantized_of(dy, ld_dy, &q, &qt), quantized_of(x, ld_x, nullptr, &xt), dtype, rows, false, st, e);
  }
  char* product = static_cast<char*>(workspace) + f.product;
  if (r == MTDAO_OK && rows > 0 && k > 0) r = launch_product(q, *wt, dx, dtype, ld_dx, 0, product, st, e);
  if (r == MTDAO_OK && n > 0 && k > 0) r = launch_product(qt, xt, dw, MTDAO_F32, ld_dw, accumulate, product, st, e);
  return r != MTDAO_OK ? r : hip_check(e, hipGetLastError(), "mtdao_linear8_backward launch");
}

}  // extern "C"
