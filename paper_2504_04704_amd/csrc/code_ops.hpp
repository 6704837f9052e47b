// 8-bit codes in registers: to and from floating point.
#pragma once
#include "attend_pass.hpp"

namespace lagkv {

typedef uint32_t u32v2_any __attribute__((ext_vector_type(2), aligned(1)));
typedef uint32_t u32v4_bytes __attribute__((ext_vector_type(4), aligned(1)));

// Four codes as numbers of binary16 or bf16 (to_half, to_bf16), or of fp32 (to_float): all of them are exact.
template <int CODE>
struct Code;
template <>
struct Code<LAGKV_CODE_INT8> {
  // Four codes as binary16: with 128 added, a code is the low byte of a number between 1024 and 1279 (a way from bytes to binary16 published by Kim et al.,
  // "Who Says Elephants Can't Run", 2022).
  static __device__ __forceinline__ void to_half(uint32_t w, uint32_t& lo, uint32_t& hi) {
    const uint32_t u = w ^ 0x80808080u;
    const f16x2 k = {(_Float16)1152.f, (_Float16)1152.f};
    lo = __builtin_bit_cast(uint32_t, __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(0x64646464u, u, 0x04010400u)) - k);
    hi = __builtin_bit_cast(uint32_t, __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(0x64646464u, u, 0x04030402u)) - k);
  }
  static __device__ __forceinline__ void to_float(uint32_t w, float* x) {
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = (float)(int8_t)(w >> (8 * i));
  }
  // (Eight bits and a sign are the upper half of an fp32.  The compiler, which would take bytes apart where they are loaded and hold one in a register each, is not to know
  // where the word comes from.)
  static __device__ __forceinline__ void to_bf16(uint32_t w, uint32_t& lo, uint32_t& hi) {
    asm("" : "+v"(w));
    float x[4];
    to_float(w, x);
    lo = __builtin_amdgcn_perm(__float_as_uint(x[1]), __float_as_uint(x[0]), 0x07060302u);
    hi = __builtin_amdgcn_perm(__float_as_uint(x[3]), __float_as_uint(x[2]), 0x07060302u);
  }
};
template <>
struct Code<LAGKV_CODE_E4M3> {
  static __device__ __forceinline__ void to_half(uint32_t w, uint32_t& lo, uint32_t& hi) {
    lo = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.f, false));
    hi = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.f, true));
  }
  static __device__ __forceinline__ void to_bf16(uint32_t w, uint32_t& lo, uint32_t& hi) {
    lo = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.f, false));
    hi = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.f, true));
  }
  static __device__ __forceinline__ void to_float(uint32_t w, float* x) {
    const auto a = __builtin_amdgcn_cvt_pk_f32_fp8(w, false), b = __builtin_amdgcn_cvt_pk_f32_fp8(w, true);
    x[0] = a[0];
    x[1] = a[1];
    x[2] = b[0];
    x[3] = b[1];
  }
};

// The type that K's codes and q go into their product in: q's own, or for fp32 bf16, of which three numbers hold all of its bits.  (V's and the weights' is binary16.)
template <int DT>
constexpr int kKeyType = DT == LAGKV_F16 ? LAGKV_F16 : LAGKV_BF16;
template <int CODE, int DT>
__device__ __forceinline__ void codes_as(uint32_t w, uint32_t& lo, uint32_t& hi) {
  if constexpr (DT == LAGKV_F16) Code<CODE>::to_half(w, lo, hi);
  else Code<CODE>::to_bf16(w, lo, hi);
}

// x less the first or the second of two numbers of binary16, in one instruction.  (It reads registers alone, and x has been read by the conversion
// that h comes from: the compiler, which does not look into it, has no wait to put before it.)
__device__ __forceinline__ float less_first(float x, uint32_t h) {
  float y;
  asm("v_fma_mix_f32 %0, %1, -1.0, %2 op_sel_hi:[1,0,0]" : "=v"(y) : "v"(h), "v"(x));
  return y;
}
__device__ __forceinline__ float less_second(float x, uint32_t h) {
  float y;
  asm("v_fma_mix_f32 %0, %1, -1.0, %2 op_sel:[1,0,0] op_sel_hi:[1,0,0]" : "=v"(y) : "v"(h), "v"(x));
  return y;
}
// A weight goes into the product with V as two numbers of binary16, its leading bits and the rest rounded, 22 bits in all, whatever the type of the outputs.  (As
// one number, 2^-12 of the sum of the weighted values' sizes may be lost: where these cancel that is more than the rounding of an output in bf16, and
// more than attend of the same rows loses.)  Half of what AElem<LAGKV_F16>::split takes: codes are never infinite, and the rest may be 0.
constexpr int kWeightParts = 2;
__device__ __forceinline__ void split_weights(float x, float y, uint32_t (&part)[kWeightParts]) {
  part[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_pkrtz(x, y));
  part[1] = AElem<LAGKV_F16>::pack(less_first(x, part[0]), less_second(y, part[0]));
}

}  // namespace lagkv
