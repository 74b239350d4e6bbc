// Device side of the types that the operators over heads take, and the layout of the 4-bit cache's blocks.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "planner.hpp"

namespace ocn {

typedef _Float16 f16;
typedef __bf16 bf16;
typedef f16 f16x2 __attribute__((ext_vector_type(2)));
typedef f16 f16x8 __attribute__((ext_vector_type(8)));
typedef bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x8 __attribute__((ext_vector_type(8), aligned(16)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

template <class T> struct Eight;
template <> struct Eight<f16> { typedef f16x8 V; };
template <> struct Eight<bf16> { typedef bf16x8 V; };
template <> struct Eight<float> { typedef f32x8 V; };

__device__ __forceinline__ uint32_t fast_quotient(uint32_t n, const FastDiv &f) { return (__umulhi(n, f.m) + n) >> f.s; }

__device__ __forceinline__ int64_t load_index(const char *p, bool wide) { return wide ? *(const int64_t *)p : (int64_t)*(const int32_t *)p; }

// any of the three types as a float
__device__ __forceinline__ float load_as_float(const char *p, int dtype) {
  if (dtype == OCN_FLOAT) return *(const float *)p;
  if (dtype == OCN_HALF) return (float)*(const f16 *)p;
  return (float)*(const bf16 *)p;
}
__device__ __forceinline__ void store_from_float(char *p, int dtype, float v) {
  if (dtype == OCN_FLOAT) *(float *)p = v;
  else if (dtype == OCN_HALF) *(f16 *)p = (f16)v;
  else *(bf16 *)p = (bf16)v;
}

// ---- a block of the cache: bytes of its parts for P tokens of D channels (a power of two) ------------
__device__ __forceinline__ int block_k_codes(int page, int d, int token, int channel) { return token * (d / 2) + channel / 2; }
__device__ __forceinline__ int block_v_codes(int page, int d, int token, int channel) {
  const int log2 = 27 - __builtin_clz(d), j = channel >> log2;         // a lane of attention has D/16 channels
  return page * (d / 2) + (((((token >> 2) * 16 + j) * 4 + (token & 3)) << log2) >> 1) + ((channel & ((1 << log2) - 1)) >> 1);
}
__device__ __forceinline__ int block_scale(int page, int d, bool v, int group, int token) {
  return page * d + 2 * (((v ? d / 32 : 0) + group) * page + token);
}

}  // namespace ocn
