// Elements of the operators' tensors: 16 bytes at a time, from any address that is aligned to an element.
//
// Rows of odd length and tensors that start anywhere are common (a slice of a flat gradient buffer), and the memory system takes
// a 16-byte access at any address: there is one path for aligned and unaligned tensors.
#ifndef CHM_ELEMENTS_H
#define CHM_ELEMENTS_H
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/chm_operators.h"

namespace chm_elements {

#define CHM_GLOBAL __attribute__((address_space(1)))
typedef uint32_t Words __attribute__((ext_vector_type(4)));
typedef uint32_t WordsAnywhere __attribute__((ext_vector_type(4), aligned(2)));

__device__ __forceinline__ float bf16_up(uint32_t u) { return __builtin_bit_cast(float, u << 16); }
__device__ __forceinline__ float f16_up(uint32_t u) { return (float)__builtin_bit_cast(_Float16, (uint16_t)u); }
__device__ __forceinline__ uint32_t bf16_down(float f) { return __builtin_bit_cast(uint16_t, (__bf16)f); }
__device__ __forceinline__ uint32_t f16_down(float f) { return __builtin_bit_cast(uint16_t, (_Float16)f); }

__device__ __forceinline__ Words load16(const char *p) { return *(const CHM_GLOBAL WordsAnywhere *)p; }
__device__ __forceinline__ void store16(char *p, Words x) { *(CHM_GLOBAL WordsAnywhere *)p = x; }
// past the caches: for results that are larger than they are (lookup of 16,384 rows of 8 KiB: 44 us with store16, 30 with this)
__device__ __forceinline__ void store16_past(char *p, Words x) { __builtin_nontemporal_store((WordsAnywhere)x, (CHM_GLOBAL WordsAnywhere *)p); }

// The N values of 16 bytes as float32, and back
template <int DT> struct Lane;
template <> struct Lane<CHM_F32> {
  enum { N = 4, SIZE = 4 };
  static __device__ __forceinline__ void up(Words x, float *v) {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = __uint_as_float(x[i]);
  }
  static __device__ __forceinline__ Words down(const float *v) {
    Words x;
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = __float_as_uint(v[i]);
    return x;
  }
  static __device__ __forceinline__ float one(const char *p) { return *(const CHM_GLOBAL float *)p; }
  static __device__ __forceinline__ void put(char *p, float v) { *(CHM_GLOBAL float *)p = v; }
};
template <> struct Lane<CHM_BF16> {
  enum { N = 8, SIZE = 2 };
  static __device__ __forceinline__ void up(Words x, float *v) {
#pragma unroll
    for (int i = 0; i < 4; ++i) { v[2 * i] = bf16_up(x[i] & 0xffffu); v[2 * i + 1] = __builtin_bit_cast(float, x[i] & 0xffff0000u); }
  }
  static __device__ __forceinline__ Words down(const float *v) {
    Words x;
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = bf16_down(v[2 * i]) | (bf16_down(v[2 * i + 1]) << 16);
    return x;
  }
  static __device__ __forceinline__ float one(const char *p) { return bf16_up(*(const CHM_GLOBAL uint16_t *)p); }
  static __device__ __forceinline__ void put(char *p, float v) { *(CHM_GLOBAL uint16_t *)p = (uint16_t)bf16_down(v); }
};
template <> struct Lane<CHM_F16> {
  enum { N = 8, SIZE = 2 };
  static __device__ __forceinline__ void up(Words x, float *v) {
#pragma unroll
    for (int i = 0; i < 4; ++i) { v[2 * i] = f16_up(x[i] & 0xffffu); v[2 * i + 1] = f16_up(x[i] >> 16); }
  }
  static __device__ __forceinline__ Words down(const float *v) {
    Words x;
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = f16_down(v[2 * i]) | (f16_down(v[2 * i + 1]) << 16);
    return x;
  }
  static __device__ __forceinline__ float one(const char *p) { return f16_up(*(const CHM_GLOBAL uint16_t *)p); }
  static __device__ __forceinline__ void put(char *p, float v) { *(CHM_GLOBAL uint16_t *)p = (uint16_t)f16_down(v); }
};

}  // namespace chm_elements
#endif
