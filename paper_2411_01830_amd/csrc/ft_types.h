// Element types of the operators' tensors in device code, and the matrix instruction on them.
#pragma once
#include <hip/hip_runtime.h>

namespace ft {

typedef float Floats4 __attribute__((ext_vector_type(4)));
typedef uint32_t Words4 __attribute__((ext_vector_type(4)));

// Vectors at any element's address: the memory pipeline splits what straddles.
struct __attribute__((packed, aligned(2))) Loose4 {
  uint32_t w[4];
};

// Global memory said to be that: a pointer that has been through an empty asm statement would be taken for one to anything.
typedef const __attribute__((address_space(1))) char *Global;
__device__ inline Global global(const void *p) { return reinterpret_cast<Global>(reinterpret_cast<uintptr_t>(p)); }

__device__ inline Words4 load16(Global p) {
  typedef const __attribute__((address_space(1))) Loose4 *P;
  return Words4{((P)p)->w[0], ((P)p)->w[1], ((P)p)->w[2], ((P)p)->w[3]};
}
__device__ inline Words4 load16(const void *p) { return load16(global(p)); }

// mfma(a, b, c) = c + a b for a of 16 x 32 and b of 32 x 16: lane l holds row l % 16 of a and column l % 16 of b, of both the
// elements 8 (l / 16) .. + 7 of the 32 (any numbering of the 32 will do, if a's and b's are the same), and of the result column l % 16, rows 4 (l / 16) .. + 3.
struct Bf16 {
  static __device__ float to_float(uint16_t v) { return __uint_as_float((uint32_t)v << 16); }
  // to the nearest, ties to even; NaN stays NaN
  static __device__ uint16_t from_float(float f) { return __builtin_bit_cast(uint16_t, (__bf16)f); }
  static __device__ uint32_t pack(float lo, float hi) {
    typedef float F __attribute__((ext_vector_type(2)));
    typedef __bf16 V __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((F{lo, hi}), V));
  }
  // towards zero (a NaN may become an infinity)
  static __device__ uint32_t pack_cut(float lo, float hi) { return __builtin_amdgcn_perm(__float_as_uint(hi), __float_as_uint(lo), 0x07060302); }
  static constexpr uint32_t kTiny = 0x0080;  // a number too small for any sum beside ones: here the smallest of full precision
  static constexpr uint32_t kExponent = 0x7f80, kLowest = 0x0080;  // an exponent of all ones (infinite or NaN), its lowest bit
  static __device__ Floats4 mfma(Words4 a, Words4 b, Floats4 c) {
    typedef __bf16 V __attribute__((ext_vector_type(8)));
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(V, a), __builtin_bit_cast(V, b), c, 0, 0, 0);
  }
};

struct Fp16 {
  static __device__ float to_float(uint16_t v) { return (float)__builtin_bit_cast(_Float16, v); }
  static __device__ uint16_t from_float(float f) { return __builtin_bit_cast(uint16_t, (_Float16)f); }
  static __device__ uint32_t pack(float lo, float hi) {
    typedef float F __attribute__((ext_vector_type(2)));
    typedef _Float16 V __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((F{lo, hi}), V));
  }
  static __device__ uint32_t pack_cut(float lo, float hi) { return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_pkrtz(lo, hi)); }
  static constexpr uint32_t kTiny = 0x0001;  // (2^-24)
  static constexpr uint32_t kExponent = 0x7c00, kLowest = 0x0400;
  static __device__ Floats4 mfma(Words4 a, Words4 b, Floats4 c) {
    typedef _Float16 V __attribute__((ext_vector_type(8)));
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(V, a), __builtin_bit_cast(V, b), c, 0, 0, 0);
  }
};

}  // namespace ft
