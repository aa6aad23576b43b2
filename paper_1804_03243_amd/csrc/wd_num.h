// Device-side helpers of the operators that make log-likelihoods: element types,
// loads and stores of the alignment of one element.
#pragma once

#include "wd_block.h"

namespace wd {

// N consecutive elements as one access with the alignment of one element (the
// hardware takes wide accesses at any address of that alignment).
template <class T, int N>
struct __attribute__((packed, aligned(sizeof(T)))) Few {
  T v[N];
};

struct Half {  // IEEE binary16
  uint16_t u;
  __device__ __forceinline__ float f() const { return (float)__builtin_bit_cast(_Float16, u); }
  static __device__ __forceinline__ Half of(float x) { return {__builtin_bit_cast(uint16_t, (_Float16)x)}; }
};
struct Bf16 {
  uint16_t u;
  __device__ __forceinline__ float f() const { return __uint_as_float((uint32_t)u << 16); }
  static __device__ __forceinline__ Bf16 of(float x) { return {__builtin_bit_cast(uint16_t, (__bf16)x)}; }
};
struct F32 {
  float u;
  __device__ __forceinline__ float f() const { return u; }
  static __device__ __forceinline__ F32 of(float x) { return {x}; }
};

}  // namespace wd
