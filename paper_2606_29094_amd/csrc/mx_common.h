// 4-bit operands: groups of 32 consecutive values of a row, one scale byte e for
// each group (the scale 2^(e - 127); 255: every value of the group is NaN) and a
// 4-bit code for each value: a sign and one of 0, 0.5, 1, 1.5, 2, 3, 4, 6. Element
// 2i of a row is the low half of its byte i. A code times its scale is exact in
// bf16 and in fp32 (at most two significant bits), and gfx950 converts two codes
// with their scale in one instruction (v_cvt_scalef32_pk_bf16_fp4, which reads the
// scale's exponent field and gives NaN for 255), so the products below multiply
// the values themselves: nothing is rounded between the stored codes and the
// matrix cores.
#pragma once

#include "common.h"

namespace dlm {

constexpr int kMxGroup = 32;

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

// the scale operand of the conversions for a scale byte
__device__ __forceinline__ float mx_scale(uint32_t e) { return __uint_as_float(e << 23); }

// eight codes (one dword, in element order) -> bf16
__device__ __forceinline__ bf16x8 mx_bf16x8(uint32_t w, float s) {
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 0);
  const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 1);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 2);
  const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 3);
  return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// Four dwords of each of the four 16-lane groups, transposed: lane l of group g comes
// with dword j of row g in v[j] and leaves with dword g of row j.
__device__ __forceinline__ u32x4 transpose_groups(u32x4 v) {
  typedef uint32_t pair __attribute__((ext_vector_type(2)));
  auto swap32 = [](uint32_t& a, uint32_t& b) {   // upper half of a with the lower one of b
    const pair r = __builtin_amdgcn_permlane32_swap(a, b, false, false);
    a = r[0], b = r[1];
  };
  auto swap16 = [](uint32_t& a, uint32_t& b) {   // odd groups of a with the even ones of b
    const pair r = __builtin_amdgcn_permlane16_swap(a, b, false, false);
    a = r[0], b = r[1];
  };
  uint32_t a = v[0], b = v[1], c = v[2], d = v[3];
  swap32(a, c);
  swap32(b, d);
  swap16(a, b);
  swap16(c, d);
  return u32x4{a, b, c, d};
}

// A block's LDS written before is seen by its other waves; loads from memory stay in
// flight.
__device__ __forceinline__ void lds_barrier() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

// Scale byte of a group from the largest magnitude's bits (any value's bits without
// the sign, compared as integers: NaN and infinity come out above every number).
// e is the exponent that puts the largest magnitude into (3.5, 7] scales, so it
// rounds to 4 or 6 and no value is off by more than one step. The
// ends are clamped so that every code times the scale is a normal number: below
// 2^-126 nothing is kept, and the top scale stays at 2^125.
__device__ __forceinline__ uint32_t mx_scale_byte(uint32_t amax) {
  if (amax >= 0x7f800000u) return 255u;
  const int e = (int)(amax >> 23) - 2 + ((amax & 0x7fffffu) > 0x600000u ? 1 : 0);
  return (uint32_t)min(max(e, 2), 252);
}

// four values -> 16 bits of codes, round to nearest (ties to the even code)
__device__ __forceinline__ uint32_t mx_codes4(float a, float b, float c, float d, float s) {
  uint32_t r = 0;
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, a, b, s, 0);
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, c, d, s, 1);
  return r & 0xffffu;
}

// fp32 x as the sum of three bf16 terms, which together hold its 24 bits: products
// of 4-bit values with fp32 ones run on the bf16 matrix cores, exactly to each term.
// Infinities and NaN go into the first term alone. The first term is rounded (a finite
// value that would round to an infinity, from 3.396e38 on, is cut off), the second cut
// off, so the sum of the first two does not overflow either; what is left after it, at
// most 8 bits, is the third.
__device__ __forceinline__ void split3(float x, bf16& hi, bf16& mid, bf16& lo) {
  auto cut = [](float v) { return __uint_as_float(__float_as_uint(v) & 0xffff0000u); };
  const uint32_t mag = __float_as_uint(x) & 0x7fffffffu;
  hi = (bf16)(mag >= 0x7f7f8000u && mag < 0x7f800000u ? cut(x) : x);
  float r = x - (float)hi;
  r = __builtin_isfinite(r) ? r : 0.f;
  mid = (bf16)cut(r);
  lo = (bf16)(r - (float)mid);
}

}  // namespace dlm
