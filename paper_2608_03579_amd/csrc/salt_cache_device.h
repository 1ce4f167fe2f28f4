// Device-side helpers of the kernels that read the paged 8-bit cache by matrix instructions
// (salt_attend.hip, salt_marks.hip): codes to bf16, operands in bf16 terms, rows over lanes.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "salt_device.h"
#include "salt_serve.h"

namespace salt {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kNegInf = -__builtin_inff();

__device__ __forceinline__ f32x4 mma_bf16(const uint4& a, const uint4& b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0,
                                                 0);
}

// Four codes (a word) as bf16, in order.
template <int FMT>
__device__ __forceinline__ uint2 codes_bf16(uint32_t w) {
  if constexpr (FMT == kKvInt8) {
    float f[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) f[e] = (float)((int)(w << (24 - 8 * e)) >> 24);
    return make_uint2(pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3]));
  } else {
    return make_uint2(__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, false)),
                      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, true)));
  }
}

template <int N>   // words
__device__ __forceinline__ void load_words(const uint8_t* p, uint32_t (&w)[N]) {
  if constexpr (N == 1) {
    w[0] = *reinterpret_cast<const uint32_t*>(p);
  } else if constexpr (N == 2) {
    const uint2 a = *reinterpret_cast<const uint2*>(p);
    w[0] = a.x; w[1] = a.y;
  } else {
#pragma unroll
    for (int j = 0; j < N; j += 4) {
      const uint4 a = *reinterpret_cast<const uint4*>(p + 4 * j);
      w[j] = a.x; w[j + 1] = a.y; w[j + 2] = a.z; w[j + 3] = a.w;
    }
  }
}

// x[8] as NT bf16 terms whose sum is x (NT = 1: rounded).
template <int NT>
__device__ __forceinline__ void split_terms(const float (&x)[8], uint4 (&o)[NT]) {
  float r[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) r[e] = x[e];
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    o[n] = make_uint4(pack_bf16x2(r[0], r[1]), pack_bf16x2(r[2], r[3]), pack_bf16x2(r[4], r[5]), pack_bf16x2(r[6], r[7]));
    if (n + 1 < NT) {
      float b[8];
      Ops<uint16_t>::to_f32(o[n], b);
#pragma unroll
      for (int e = 0; e < 8; ++e) r[e] -= b[e];
    }
  }
}

// Over the four lanes of a row (l, l ^ 16, l ^ 32, l ^ 48): halves and then rows of 16 lanes
// change places, without LDS.
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ float row_max(float v) {
  u32x2 w = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = fmaxf(__uint_as_float(w[0]), __uint_as_float(w[1]));
  w = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(w[0]), __uint_as_float(w[1]));
}
__device__ __forceinline__ float row_sum(float v) {
  u32x2 w = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = __uint_as_float(w[0]) + __uint_as_float(w[1]);
  w = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(w[0]) + __uint_as_float(w[1]);
}
// The running maximum follows a row's largest logit only when that is this much above it
// (log2): exponentials stay below 2^8, and sums and products are seldom scaled anew.
constexpr float kMaxSlack = 8.f;

// Word i of p, for a wave-uniform i: by way of the scalar unit.  (p is not written by this launch.)
__device__ __forceinline__ int uniform_word(const int32_t* p, int i) {
  return ((const __attribute__((address_space(4))) int32_t*)(uintptr_t)p)[__builtin_amdgcn_readfirstlane(i)];
}

// A lane's offset from a uniform base, kept as such: otherwise the compiler adds it to the loop's fixed part
// of the base ahead of the loop, two registers for every load in it.
__device__ __forceinline__ uint32_t lane_offset(uint32_t v) {
  asm volatile("" : "+v"(v));
  return v;
}

// The instruction itself: fmaxf first quiets every operand, which might be a signalling NaN.
__device__ __forceinline__ float max3_of(float a, float b, float c) {
  float r;
  asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
  return r;
}

template <typename E>
__device__ __forceinline__ void load8(const E* p, float (&v)[8]) { Ops<E>::to_f32(Ops<E>::load(p), v); }

}  // namespace salt
