// Element types of the operators' tensors in device code.
#pragma once
#include <hip/hip_bf16.h>
#include <hip/hip_fp16.h>
#include <hip/hip_runtime.h>

namespace ft {

struct Bf16 {
  static __device__ float to_float(uint16_t v) { return __uint_as_float((uint32_t)v << 16); }
  // to the nearest, ties to even; NaN stays NaN
  static __device__ uint16_t from_float(float f) { return __builtin_bit_cast(uint16_t, (__bf16)f); }
};

struct Fp16 {
  static __device__ float to_float(uint16_t v) { return (float)__builtin_bit_cast(_Float16, v); }
  static __device__ uint16_t from_float(float f) { return __builtin_bit_cast(uint16_t, (_Float16)f); }
};

}  // namespace ft
