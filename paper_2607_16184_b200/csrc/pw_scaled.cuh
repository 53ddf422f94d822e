// Element types and the scaled 8-bit format, shared by the kernels that write it and the product that reads it:
// e4m3 codes (largest value 448) with an fp32 scale per block of 128 columns and 1 or 128 rows.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <stdint.h>

#include <type_traits>

#include "pw_common.cuh"

namespace pw {

constexpr float kE4m3Max = 448.0f;
constexpr float kMinScale = 1.17549435e-38f;    // 2^-126: the smallest scale whose reciprocal is finite

inline bool type_ok(int t) { return t == PW_F32 || t == PW_F16 || t == PW_BF16; }
inline int type_size(int t) { return t == PW_F32 ? 4 : 2; }
inline bool is_aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }
// Last check before a launch: the context's status word and multiprocessor count belong to the device it was made on.
inline pw_status check_device(const pw_ctx* ctx) {
  int dev = -1;
  PW_CUDA_OK(cudaGetDevice(&dev));
  return dev == ctx->device ? PW_OK : PW_ERR_INVALID_ARG;
}

// Scale of a block whose largest magnitude is `top`.  A block of zeros keeps scale 1; a block so small that the
// reciprocal of its scale would overflow takes the smallest usable scale.
__device__ __forceinline__ float block_scale(float top) {
  return top == 0.f ? 1.f : fmaxf(__fdiv_rn(top, kE4m3Max), kMinScale);
}
// Two codes, the first in the low byte; values beyond 448 (by the rounding of the scale) become 448, NaN stays NaN.
__device__ __forceinline__ uint32_t pack_e4m3(float lo, float hi) {
  uint16_t r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
  return r;
}
__device__ __forceinline__ float abs_max(float m, float v) { return fmaxf(m, fabsf(v)); }

__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(__half v) { return __half2float(v); }
__device__ __forceinline__ float to_f32(__nv_bfloat16 v) { return __bfloat162float(v); }
template <class T>
__device__ __forceinline__ T from_f32(float v) {          // to nearest, ties to even
  if constexpr (std::is_same<T, float>::value) return v;
  else if constexpr (std::is_same<T, __half>::value) return __float2half_rn(v);
  else return __float2bfloat16_rn(v);
}

// Eight consecutive elements as they lie in memory (16 or 32 bytes): loads of several of these stay in flight
// together, the conversion comes afterwards.
template <class T>
struct Raw8 {
  uint4 a;
  __device__ __forceinline__ void load(const T* p) { a = *reinterpret_cast<const uint4*>(p); }
  __device__ __forceinline__ void zero() { a = make_uint4(0, 0, 0, 0); }
  // keeps the compiler from holding on to values it has converted before
  __device__ __forceinline__ void forget() { asm volatile("" : "+r"(a.x), "+r"(a.y), "+r"(a.z), "+r"(a.w)); }
  __device__ __forceinline__ void get(float* v) const {
    const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (sizeof(T) == 2 && std::is_same<T, __half>::value) {
        const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
        v[2 * i] = f.x;
        v[2 * i + 1] = f.y;
      } else {
        v[2 * i] = __uint_as_float(w[i] << 16);
        v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
      }
    }
  }
};
template <>
struct Raw8<float> {
  float4 a, b;
  __device__ __forceinline__ void load(const float* p) {
    a = reinterpret_cast<const float4*>(p)[0];
    b = reinterpret_cast<const float4*>(p)[1];
  }
  __device__ __forceinline__ void zero() { a = b = make_float4(0.f, 0.f, 0.f, 0.f); }
  __device__ __forceinline__ void forget() {}
  __device__ __forceinline__ void get(float* v) const {
    v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w;
    v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
  }
};

__device__ __forceinline__ uint32_t pack_half(float lo, float hi) {
  const __half2 h = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ uint32_t pack_bf(float lo, float hi) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}
// Eight consecutive values, each rounded once to the type (aligned store).
__device__ __forceinline__ void store8(void* base, int64_t at, int type, const float* v) {
  if (type == PW_F32) {
    float4* p = reinterpret_cast<float4*>(static_cast<float*>(base) + at);
    p[0] = make_float4(v[0], v[1], v[2], v[3]);
    p[1] = make_float4(v[4], v[5], v[6], v[7]);
  } else if (type == PW_F16) {
    *reinterpret_cast<uint4*>(static_cast<__half*>(base) + at) =
        make_uint4(pack_half(v[0], v[1]), pack_half(v[2], v[3]), pack_half(v[4], v[5]), pack_half(v[6], v[7]));
  } else {
    *reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(base) + at) =
        make_uint4(pack_bf(v[0], v[1]), pack_bf(v[2], v[3]), pack_bf(v[4], v[5]), pack_bf(v[6], v[7]));
  }
}
__device__ __forceinline__ void store1(void* base, int64_t at, int type, float v) {
  if (type == PW_F32) static_cast<float*>(base)[at] = v;
  else if (type == PW_F16) static_cast<__half*>(base)[at] = __float2half_rn(v);
  else static_cast<__nv_bfloat16*>(base)[at] = __float2bfloat16_rn(v);
}
__device__ __forceinline__ float load1(const void* base, int64_t at, int type) {
  if (type == PW_F32) return static_cast<const float*>(base)[at];
  if (type == PW_F16) return __half2float(static_cast<const __half*>(base)[at]);
  return __bfloat162float(static_cast<const __nv_bfloat16*>(base)[at]);
}

}  // namespace pw
