// Device and launch helpers of the token models' kernels (HIP only).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "internal.h"
#include "tokens.h"

namespace nbsgd {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
// 16 bytes at the alignment of an element: one dwordx4 access all the same (gfx950
// takes unaligned vector accesses), a few more cache lines where it straddles them
typedef uint32_t u32x4_any __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t u32x2_any __attribute__((ext_vector_type(2), aligned(2)));

__device__ __forceinline__ float bf16_lo(uint32_t v) { return __builtin_bit_cast(float, v << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t v) {
  return __builtin_bit_cast(float, v & 0xffff0000u);
}
// two floats to bf16, nearest even (one v_cvt_pk_bf16_f32)
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2){lo, hi}, bf16x2));
}

// Orders the wave's LDS writes before its later accesses to other lanes' data.
__device__ __forceinline__ void wave_fence() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// An activation element type: V of them fill 16 bytes.
template <typename T>
struct Elem;
template <>
struct Elem<float> {
  static constexpr int V = 4;
  static __device__ __forceinline__ float load(const float* p) { return *p; }
  static __device__ __forceinline__ void store(float* p, float v) { *p = v; }
  static __device__ __forceinline__ void expand(u32x4 r, float (&v)[4]) {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const uint32_t w = r[k];  // a cast of the vector's element itself would take element 0
      v[k] = __builtin_bit_cast(float, w);
    }
  }
  static __device__ __forceinline__ u32x4 collapse(const float (&v)[4]) {
    u32x4 r;
#pragma unroll
    for (int k = 0; k < 4; ++k) r[k] = __builtin_bit_cast(uint32_t, v[k]);
    return r;
  }
};
template <>
struct Elem<__bf16> {
  static constexpr int V = 8;
  static __device__ __forceinline__ float load(const __bf16* p) { return (float)*p; }
  static __device__ __forceinline__ void store(__bf16* p, float v) { *p = (__bf16)v; }
  static __device__ __forceinline__ void expand(u32x4 r, float (&v)[8]) {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      v[2 * k] = bf16_lo(r[k]);
      v[2 * k + 1] = bf16_hi(r[k]);
    }
  }
  static __device__ __forceinline__ u32x4 collapse(const float (&v)[8]) {
    u32x4 r;
#pragma unroll
    for (int k = 0; k < 4; ++k) r[k] = pack2(v[2 * k], v[2 * k + 1]);
    return r;
  }
};

// The first `n` (at least one, V of them at most) elements at p as 16 bytes, zeros behind them.
__device__ __forceinline__ u32x4 load16(const float* p, int n) {
  if (n >= 4) return *reinterpret_cast<const u32x4_any*>(p);
  uint32_t w[4] = {0u, 0u, 0u, 0u};
#pragma unroll
  for (int k = 0; k < 4; ++k)
    if (k < n) w[k] = __builtin_bit_cast(uint32_t, p[k]);
  return (u32x4){w[0], w[1], w[2], w[3]};
}
// The short ones read the last element over and over: behind branches the halves of a word
// wait for each other.
__device__ __forceinline__ u32x4 load16(const __bf16* p, int n) {
  if (n >= 8) return *reinterpret_cast<const u32x4_any*>(p);
  __bf16 v[8];
#pragma unroll
  for (int k = 0; k < 8; ++k) v[k] = p[min(k, n - 1)];
  uint32_t w[4] = {0u, 0u, 0u, 0u};
#pragma unroll
  for (int k = 0; k < 8; ++k)
    w[k / 2] |= k < n ? (uint32_t)__builtin_bit_cast(uint16_t, v[k]) << (16 * (k % 2)) : 0u;
  return (u32x4){w[0], w[1], w[2], w[3]};
}
template <typename T>
__device__ __forceinline__ void store16(T* p, u32x4 r, int n) {
  constexpr int V = Elem<T>::V, per = V / 4;
  if (n >= V) {
    *reinterpret_cast<u32x4_any*>(p) = r;
    return;
  }
  const uint32_t w[4] = {r[0], r[1], r[2], r[3]};
#pragma unroll
  for (int k = 0; k < V; ++k)
    if (k < n) {
      if constexpr (per == 1) p[k] = __builtin_bit_cast(float, w[k]);
      else p[k] = __builtin_bit_cast(__bf16, (uint16_t)(w[k / per] >> (16 * (k % per))));
    }
}

// Whether rows of `bytes` bytes apart lie on whole 128-byte lines.
inline bool on_lines(const void* p, int64_t bytes) { return !((uintptr_t)p & 127) && bytes % 128 == 0; }

// Refuses a stream of a device that is not the current one (kernels would be looked up on
// the wrong one).
inline nbsgd_status check_stream(void* stream) {
  if (!stream) return NBSGD_OK;
  int dev = -1;
  hipDevice_t sdev = -1;
  hipError_t e = hipGetDevice(&dev);
  if (e == hipSuccess) e = hipStreamGetDevice(reinterpret_cast<hipStream_t>(stream), &sdev);
  if (e != hipSuccess) return fail(NBSGD_E_HIP, "stream's device: %s", hipGetErrorString(e));
  if ((int)sdev != dev)
    return fail(NBSGD_E_ARG, "stream belongs to device %d but device %d is current", (int)sdev, dev);
  return NBSGD_OK;
}

inline nbsgd_status launched(const char* what) {
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return fail(NBSGD_E_HIP, "%s launch failed: %s", what, hipGetErrorString(e));
  return NBSGD_OK;
}

}  // namespace nbsgd
