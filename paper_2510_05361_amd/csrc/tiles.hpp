// Device helpers of kernels that multiply matrices in tiles: fragments, rows of
// 128 bytes in LDS, buffers, waits.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace mtdao {
namespace ops {

typedef int v8i __attribute__((ext_vector_type(8)));
typedef int v4i __attribute__((ext_vector_type(4)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef float v16f __attribute__((ext_vector_type(16)));
typedef __bf16 v2bf __attribute__((ext_vector_type(2)));
typedef __bf16 v8bf __attribute__((ext_vector_type(8)));

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

}  // namespace ops
}  // namespace mtdao
