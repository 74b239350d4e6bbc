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

// ---- rows: eight channels of a lane -------------------------------------------------------------------
constexpr int kEight = 8;
template <class T> using eight_t = typename Eight<T>::V;

// eight channels from e on; those outside the row are zero
template <class T, bool VEC> __device__ __forceinline__ eight_t<T> load_eight(const char *row, int64_t step, int e, int d) {
  if constexpr (VEC) {
    return *(const eight_t<T> *)(row + e * (int)sizeof(T));
  } else {
    eight_t<T> v;
#pragma unroll
    for (int i = 0; i < kEight; ++i) v[i] = e + i < d ? *(const T *)(row + (e + i) * step) : (T)0.0f;
    return v;
  }
}
// (stream: past the caches, for outputs that they could not keep)
template <class T, bool VEC> __device__ __forceinline__ void store_eight(char *row, int64_t step, int e, int d, const float *v, bool stream) {
  if constexpr (VEC) {
    eight_t<T> o;
#pragma unroll
    for (int i = 0; i < kEight; ++i) o[i] = (T)v[i];
    if (stream) {
      asm volatile("");     // (these keep the two apart: made into one store, they would be an ordinary one)
      __builtin_nontemporal_store(o, (eight_t<T> *)(row + e * (int)sizeof(T)));
      asm volatile("");
    } else {
      *(eight_t<T> *)(row + e * (int)sizeof(T)) = o;
    }
  } else {
#pragma unroll
    for (int i = 0; i < kEight; ++i)
      if (e + i < d) *(T *)(row + (e + i) * step) = (T)v[i];
  }
}

// ---- lanes ----------------------------------------------------------------------------------------------
template <int CTRL> __device__ __forceinline__ float other_lane(float x) {
  return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), CTRL, 0xf, 0xf, true));
}
template <int CTRL> __device__ __forceinline__ uint32_t other_lane_bits(uint32_t x) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, 0xf, 0xf, true); }
// the sum over a row's lanes (1, 2, 4 ... 64 of them): exchanges inside sixteen lanes cost no trip through LDS
__device__ __forceinline__ float sum_over_row(float v, int lanes) {
  if (lanes > 1) v += other_lane<0xb1>(v);      // 1 0 3 2
  if (lanes > 2) v += other_lane<0x4e>(v);      // 2 3 0 1
  if (lanes > 4) v += other_lane<0x141>(v);     // eight lanes mirrored
  if (lanes > 8) v += other_lane<0x140>(v);     // sixteen lanes mirrored
  if (lanes > 16) v += __shfl_xor(v, 16);
  if (lanes > 32) v += __shfl_xor(v, 32);
  return v;
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
