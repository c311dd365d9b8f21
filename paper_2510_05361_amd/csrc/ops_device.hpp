// Device helpers of the operators of include/mtdao_ops.h: storage types,
// vector accesses at element alignment, 8-bit blocks, wave reductions.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace mtdao {
namespace ops {

constexpr int kBlock8 = 128;

using bf16_t = uint16_t;

__device__ __forceinline__ float to_f32(float x) { return x; }
__device__ __forceinline__ float to_f32(bf16_t b) { return __uint_as_float((uint32_t)b << 16); }

// Two fp32 values as bf16, round to nearest even (NaN stays NaN).
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  bf16x2 v;
  v[0] = (__bf16)a;
  v[1] = (__bf16)b;
  return __builtin_bit_cast(uint32_t, v);
}

// Vectors at addresses aligned to their element only (the hardware takes
// them at any such address).
typedef float f32v4 __attribute__((ext_vector_type(4), aligned(4)));
typedef uint32_t u32v2h __attribute__((ext_vector_type(2), aligned(2)));
typedef uint32_t u32v4h __attribute__((ext_vector_type(4), aligned(2)));

template <bool NT, typename V>
__device__ __forceinline__ V vec_load(const void* p) {
  if constexpr (NT) return __builtin_nontemporal_load(reinterpret_cast<const V*>(p));
  else return *reinterpret_cast<const V*>(p);
}
template <bool NT, typename V>
__device__ __forceinline__ void vec_store(void* p, V v) {
  if constexpr (NT) __builtin_nontemporal_store(v, reinterpret_cast<V*>(p));
  else *reinterpret_cast<V*>(p) = v;
}

// N = 4 or 8 consecutive elements as fp32.
template <int N, bool NT = false>
__device__ __forceinline__ void load_full(const float* p, float (&o)[N]) {
#pragma unroll
  for (int k = 0; k < N / 4; ++k) {
    const f32v4 a = vec_load<NT, f32v4>(p + 4 * k);
#pragma unroll
    for (int t = 0; t < 4; ++t) o[4 * k + t] = a[t];
  }
}
template <int N, bool NT = false>
__device__ __forceinline__ void load_full(const bf16_t* p, float (&o)[N]) {
  uint32_t w[N / 2];
  if constexpr (N == 4) {
    const u32v2h a = vec_load<NT, u32v2h>(p);
    w[0] = a[0];
    w[1] = a[1];
  } else {
    const u32v4h a = vec_load<NT, u32v4h>(p);
#pragma unroll
    for (int t = 0; t < 4; ++t) w[t] = a[t];
  }
#pragma unroll
  for (int t = 0; t < N / 2; ++t) {
    o[2 * t] = __uint_as_float(w[t] << 16);
    o[2 * t + 1] = __uint_as_float(w[t] & 0xffff0000u);
  }
}
template <int N, bool NT = false>
__device__ __forceinline__ void store_full(float* p, const float (&o)[N]) {
#pragma unroll
  for (int k = 0; k < N / 4; ++k) {
    const f32v4 a = {o[4 * k], o[4 * k + 1], o[4 * k + 2], o[4 * k + 3]};
    vec_store<NT, f32v4>(p + 4 * k, a);
  }
}
template <int N, bool NT = false>
__device__ __forceinline__ void store_full(bf16_t* p, const float (&o)[N]) {
  if constexpr (N == 4) {
    const u32v2h a = {pack_bf16(o[0], o[1]), pack_bf16(o[2], o[3])};
    vec_store<NT, u32v2h>(p, a);
  } else {
    const u32v4h a = {pack_bf16(o[0], o[1]), pack_bf16(o[2], o[3]), pack_bf16(o[4], o[5]), pack_bf16(o[6], o[7])};
    vec_store<NT, u32v4h>(p, a);
  }
}

// The first n of N elements (n <= 0: none, n >= N: all), zeros for the rest.
template <int N, bool NT = false, typename T>
__device__ __forceinline__ void load_some(const T* p, int n, float (&o)[N]) {
  if (n >= N) {
    load_full<N, NT>(p, o);
  } else {
#pragma unroll
    for (int t = 0; t < N; ++t) o[t] = t < n ? to_f32(p[t]) : 0.0f;
  }
}
__device__ __forceinline__ void store_one(float* p, float v) { *p = v; }
__device__ __forceinline__ void store_one(bf16_t* p, float v) { *p = (bf16_t)pack_bf16(v, 0.0f); }
template <int N, bool NT = false, typename T>
__device__ __forceinline__ void store_some(T* p, int n, const float (&o)[N]) {
  if (n >= N) {
    store_full<N, NT>(p, o);
  } else {
#pragma unroll
    for (int t = 0; t < N; ++t)
      if (t < n) store_one(p + t, o[t]);
  }
}

// Eight elements as they are in memory, zeros from n on (n <= 0: none).
template <typename T, bool NT = false>
struct Raw;
template <bool NT>
struct Raw<bf16_t, NT> {
  uint32_t w[4];
  __device__ __forceinline__ void set(int i, uint32_t dword) { w[i] = dword; }
  __device__ __forceinline__ void load(const bf16_t* p, int n) {
    if (n >= 8) {
      const u32v4h v = vec_load<NT, u32v4h>(p);
#pragma unroll
      for (int t = 0; t < 4; ++t) w[t] = v[t];
    } else {
#pragma unroll
      for (int t = 0; t < 4; ++t)
        w[t] = (2 * t < n ? (uint32_t)p[2 * t] : 0u) | (2 * t + 1 < n ? (uint32_t)p[2 * t + 1] << 16 : 0u);
    }
  }
  __device__ __forceinline__ void values(float (&o)[8]) const {
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      o[2 * t] = __uint_as_float(w[t] << 16);
      o[2 * t + 1] = __uint_as_float(w[t] & 0xffff0000u);
    }
  }
};
template <bool NT>
struct Raw<float, NT> {
  float w[8];
  __device__ __forceinline__ void set(int i, uint32_t dword) { w[i] = __uint_as_float(dword); }
  __device__ __forceinline__ void load(const float* p, int n) { load_some<8, NT>(p, n, w); }
  __device__ __forceinline__ void values(float (&o)[8]) const {
#pragma unroll
    for (int t = 0; t < 8; ++t) o[t] = w[t];
  }
};

// The i-th of tokens or targets of 32 or 64 (wide) bits.
__device__ __forceinline__ int64_t id_of(const void* ids, int32_t wide, int64_t i) {
  return wide ? reinterpret_cast<const int64_t*>(ids)[i] : (int64_t) reinterpret_cast<const int32_t*>(ids)[i];
}

// A wave-uniform value that no running kernel writes, through the scalar
// cache.
template <typename T>
__device__ __forceinline__ T uniform_load(const T* p) {
  return *(const __attribute__((address_space(4))) T*)p;
}

// What lanes of a wave have written to LDS the others read behind this.  LDS serves a wave in order;
// the compiler has to keep it, and the barrier alone does not bind memory.
__device__ __forceinline__ void lanes_done() {
  __builtin_amdgcn_wave_barrier();
  asm volatile("" ::: "memory");
}

// ---------------------------------------------------------- wave reductions

// x of the lane that a DPP control names (all lanes of the row take part).
template <int CTRL>
__device__ __forceinline__ float dpp(float x) {
  return __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(x), CTRL, 0xf, 0xf, true));
}
constexpr int kRor8 = 0x128, kRor4 = 0x124, kRor2 = 0x122, kRor1 = 0x121;  // rotations within rows of 16 lanes

// x of this lane and of the lane 16 (32) away, within 32 (64) lanes: both
// lanes get the same pair in the same order.
struct Pair {
  float a, b;
};
__device__ __forceinline__ Pair with16(float x) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return {__uint_as_float(r[0]), __uint_as_float(r[1])};
}
__device__ __forceinline__ Pair with32(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return {__uint_as_float(r[0]), __uint_as_float(r[1])};
}

// Largest / sum over rows of 16 lanes, groups of 32 lanes or the wave, in
// every lane.  The order of the sums is fixed.
__device__ __forceinline__ float max16(float x) {
  x = fmaxf(x, dpp<kRor8>(x));
  x = fmaxf(x, dpp<kRor4>(x));
  x = fmaxf(x, dpp<kRor2>(x));
  return fmaxf(x, dpp<kRor1>(x));
}
__device__ __forceinline__ float max_with16(float x) {
  const Pair p = with16(x);
  return fmaxf(p.a, p.b);
}
__device__ __forceinline__ float max_with32(float x) {
  const Pair p = with32(x);
  return fmaxf(p.a, p.b);
}
__device__ __forceinline__ float max32(float x) { return max_with16(max16(x)); }
__device__ __forceinline__ float sum64(float x) {
  x += dpp<kRor8>(x);
  x += dpp<kRor4>(x);
  x += dpp<kRor2>(x);
  x += dpp<kRor1>(x);
  const Pair p = with16(x);
  const Pair q = with32(p.a + p.b);
  return q.a + q.b;
}

// ------------------------------------------------------------- 8-bit blocks

// Largest |x| so far, NaN left out.  Infinite only where an infinity was seen:
// then the maximum is formed again from finite_abs.
__device__ __forceinline__ float max_abs(float m, float x) { return fmaxf(m, fabsf(x)); }
__device__ __forceinline__ bool is_infinite(float m) { return m > 3.4028234664e38f; }
// |x| where x is finite, else 0: what a block's scale is formed from.
__device__ __forceinline__ float finite_abs(float x) {
  const float a = fabsf(x);
  return a <= 3.4028234664e38f ? a : 0.0f;  // false for NaN
}

// Byte e + 127 of the smallest 2^e with amax / 2^e <= 448 = 1.75 2^8.
__device__ __forceinline__ uint32_t scale_byte(float amax) {
  const uint32_t u = __float_as_uint(amax);
  const int e = (int)(u >> 23) - 8 + ((u & 0x7fffffu) > 0x600000u ? 1 : 0);
  return (uint32_t)(e < 1 ? 1 : e > 254 ? 254 : e);
}
// 2^e, and 2^-e (bytes 1..253, which is all that scale_byte gives: no finite
// fp32 amax exceeds 247).
__device__ __forceinline__ float scale_of(uint32_t byte) { return __uint_as_float(byte ? byte << 23 : 0x00400000u); }
__device__ __forceinline__ float inverse_scale_of(uint32_t byte) { return __uint_as_float((254u - byte) << 23); }

// Four scaled values as e4m3 codes: rounded to nearest even; infinities and
// NaN give NaN codes (a kernel's floating-point mode does not clamp).
__device__ __forceinline__ uint32_t codes_of(float a, float b, float c, float d) {
  int r = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, r, true);
}

__device__ __forceinline__ void values_of(uint32_t codes, float (&o)[4]) {
  const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)codes, false);
  const auto hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)codes, true);
  o[0] = lo[0];
  o[1] = lo[1];
  o[2] = hi[0];
  o[3] = hi[1];
}

}  // namespace ops
}  // namespace mtdao
