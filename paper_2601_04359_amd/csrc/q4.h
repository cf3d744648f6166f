// The 4-bit cache: element format, row layout and the conversions that every kernel over it shares (gfx950 only).
//
// 32 neighbouring dims of a row are a group.  A group's scale is 2^e, e the least integer with max|x| <= 7 * 2^e, so
// that the largest element is never further than half a step from its code (6 is the largest code, 7 the border up to
// which a step of 2 rounds to it); e is kept from -120 to 125, so that every value is a normal, finite bf16 number
// and codes turn into bf16 matrix operands without a rounding.  The byte of a scale is e + 127; 255 marks a group
// that held a NaN or an infinity, which reads as NaN throughout.
#pragma once

#include "common.h"

namespace pc {

typedef __attribute__((__vector_size__(2 * sizeof(__bf16)))) __bf16 bf16x2;

constexpr int kQ4MinExp = -120, kQ4MaxExp = 125;
constexpr int kQ4BadScale = 255;
constexpr int kMaxRows = 1 << 30;      // of a call over a cache

// A cache in 4 bits as the kernels see it (pc_q4_cache with the heads' strides in bytes).
struct Q4Rows {
  const uint8_t *k_codes, *k_scales, *v_codes, *v_scales;
  int64_t code_stride_h, scale_stride_h;
};

// The scale byte of a group from the bits of its largest magnitude (fp32 bits, no sign).  A value whose significand
// is above 1.75 is above 7 * 2^(exponent - 2).
__device__ __forceinline__ int q4_scale_byte(uint32_t top) {
  if (top >= 0x7f800000u) return kQ4BadScale;
  const int e = static_cast<int>(top >> 23) - 129 + ((top & 0x7fffffu) > 0x600000u);
  return min(max(e, kQ4MinExp), kQ4MaxExp) + 127;
}
// 2^e as a float, of a scale byte (255 gives an infinity's bits, which the conversion takes as NaN)
__device__ __forceinline__ float q4_scale(int byte) { return __uint_as_float(static_cast<uint32_t>(byte) << 23); }

// Eight codes (a dword, element 0 in the low half of byte 0) times 2^e as bf16; exact.
__device__ __forceinline__ bf16x8 q4_to_bf16(uint32_t codes, float scale) {
  union {
    bf16x8 all;
    bf16x2 two[4];
  } v;
  v.two[0] = __builtin_bit_cast(bf16x2, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 0));
  v.two[1] = __builtin_bit_cast(bf16x2, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 1));
  v.two[2] = __builtin_bit_cast(bf16x2, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 2));
  v.two[3] = __builtin_bit_cast(bf16x2, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 3));
  return v.all;
}

// x in 24 bits of significand as the sum of three bf16 numbers (NaN and infinities end up as NaN or the infinity in
// the first with NaN behind it: the sum is not finite either way).
__device__ __forceinline__ void split3(float x, __bf16& a, __bf16& b, __bf16& c) {
  a = static_cast<__bf16>(x);
  const float r = x - static_cast<float>(a);
  b = static_cast<__bf16>(r);
  c = static_cast<__bf16>(r - static_cast<float>(b));
}

// ---- host: what every entry point over a cache checks -----------------------------------------------
inline int check_q4_cache(const pc_q4_cache* c, int D, const char* who) {
  PC_REQUIRE(c, PC_ERR_NULL, "%s: the cache is NULL", who);
  PC_REQUIRE(c->k_codes && c->k_scales && c->v_codes && c->v_scales, PC_ERR_NULL, "%s: a pointer of the cache is NULL", who);
  const uintptr_t codes = reinterpret_cast<uintptr_t>(c->k_codes) | reinterpret_cast<uintptr_t>(c->v_codes) |
                          static_cast<uintptr_t>(c->code_stride_h);
  const uintptr_t scales = reinterpret_cast<uintptr_t>(c->k_scales) | reinterpret_cast<uintptr_t>(c->v_scales) |
                           static_cast<uintptr_t>(c->scale_stride_h);
  PC_REQUIRE(codes % 16 == 0 && scales % (D / 32) == 0, PC_ERR_SHAPE,
             "%s: codes must be 16-byte aligned, scales aligned to a row's %d bytes, strides alike", who, D / 32);
  return PC_OK;
}

// Rows row0 .. row0 + n - 1 of H heads lie within the heads' strides.
inline int check_q4_span(const pc_q4_cache* c, int H, int row0, int64_t n, int D, const char* who) {
  const int64_t end = row0 + n;
  PC_REQUIRE(H == 1 || (c->code_stride_h >= end * (D / 2) && c->scale_stride_h >= end * (D / 32)), PC_ERR_SHAPE,
             "%s: rows up to %lld do not fit the cache's head strides", who, static_cast<long long>(end));
  return PC_OK;
}

}  // namespace pc
