// What the operators of beams behind one prompt share (spd_append.cu, spd_attend.cu, spd_select.cu, spd_reorder.cu).
#pragma once
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <initializer_list>

#include "spd.h"

extern "C" int spd_internal_cuda_fail(cudaError_t e, const char *what);

namespace spd {

inline bool aligned(const void *p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }
// Whether arrays lie on whole elements of so many bytes (null ones do): the host sees to it, since a device faults on those that do not.
inline bool all_aligned(size_t a, std::initializer_list<const void *> arrays) {
  for (const void *p : arrays)
    if (!aligned(p, a)) return false;
  return true;
}
inline size_t type_bytes(int dtype) { return dtype == SPD_F32 ? 4 : 2; }
inline bool known_type(int dtype) { return dtype == SPD_F32 || dtype == SPD_BF16; }
inline int launched(const char *what) {
  const cudaError_t e = cudaGetLastError();
  return e == cudaSuccess ? SPD_OK : spd_internal_cuda_fail(e, what);
}

#ifdef __CUDACC__
__device__ __forceinline__ float to_float(float v) { return v; }
__device__ __forceinline__ float to_float(__nv_bfloat16 v) { return __bfloat162float(v); }
template <typename T> __device__ __forceinline__ T from_float(float v);
template <> __device__ __forceinline__ float from_float<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

__device__ __forceinline__ float low_bf16(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float high_bf16(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t *>(&v);
}
// 2^v, results below 2^-126 as zero.
__device__ __forceinline__ float power2(float v) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
  return r;
}
// Four neighbouring elements, aligned to their size together.
__device__ __forceinline__ float4 load4(const float *p) { return *reinterpret_cast<const float4 *>(p); }
__device__ __forceinline__ float4 load4(const __nv_bfloat16 *p) {
  const uint2 w = *reinterpret_cast<const uint2 *>(p);
  return make_float4(low_bf16(w.x), high_bf16(w.x), low_bf16(w.y), high_bf16(w.y));
}
__device__ __forceinline__ void store4(float *p, const float4 &v) { *reinterpret_cast<float4 *>(p) = v; }
__device__ __forceinline__ void store4(__nv_bfloat16 *p, const float4 &v) {
  *reinterpret_cast<uint2 *>(p) = make_uint2(pack_bf16(v.x, v.y), pack_bf16(v.z, v.w));
}
#endif

}  // namespace spd
