// Microscaled (MX) operands: blocks of 32 elements along the contraction share one power of two (E8M0, a byte: exponent + 127).
//
// An element is one E2M1 code h, x ~ s h (4 bits), or two, x ~ s (h + l / 8) (8 bits): h the nearest code to x / s, l the nearest to
// what is left at an eighth of the scale.  8 bits are two codes and not one E4M3 code because the matrix cores lose bits of 8-bit
// products: beside a large product of the same instruction the small ones are cut off at 2^-13 or so of it (measured, normal data: 5e-6
// of the result with one E4M3 operand, 1.5e-5 with two), while products of E2M1 codes come out exactly; two 4-bit instructions take as
// long as one 8-bit one; and a uniform grid of sixteenths keeps more of the values: 37.5 dB on normal data (E4M3: 31.5), 34.8 on
// Student-t with three degrees of freedom.
//
// A line's codes take pitch(length) elements, length rounded up to 512: a line of codes begins at a multiple of 256 bytes, its scales at
// a multiple of 16, and no kernel meets a line's end inside a load.  What lies behind `length` is the code 0 under a finite scale.  The
// second codes lie in a plane of their own behind the first, so that either plane is an operand of the matrix instruction.
//
// Scale of a block with largest magnitude m: the smallest power of two with m <= 7 s.  Magnitudes up to 7 s have 6 s as their nearest
// value on the grid carried on beyond 6, so what saturates errs by no more than the grid's own half step.  Normal data keep 19.0 dB in 4
// bits (rule 2^(floor(log2 m) - 2): 18.8; smallest s with m <= 6 s: 18.7), Student-t 17.6 (17.4; 17.0).
// Exponents are held in [-126, 127] (8 bits: [-123, 127], so that an eighth is a normal number as well); a block with an infinity or a
// NaN gets the byte 255, which stands for NaN in the matrix instruction and in the decode alike.
#pragma once
#include "fp4_common.h"

constexpr int MX_BLOCK = 32;
constexpr int MX_PITCH = 512;
FP4_HD int64_t mx_pitch_of(int64_t length) { return (length + MX_PITCH - 1) / MX_PITCH * MX_PITCH; }

// Byte of the scale of a block from the bits of its largest magnitude (as fp32; a NaN's bits are larger than any number's).
template <int BITS>
FP4_HD uint32_t mx_scale_byte(uint32_t amax_bits) {
  constexpr int32_t least = BITS == 4 ? 1 : 4;
  const int32_t e = (int32_t)((amax_bits + 0x1fffffu) >> 23) - 2;   // mantissas over 1.75 carry into the exponent
  return amax_bits >= 0x7f800000u ? 255u : (uint32_t)(e < least ? least : e);
}
constexpr uint32_t MX_EIGHTH = 0x03030303u;   // four scales less this: an eighth of each

#if defined(__HIPCC__)
typedef __bf16 mx_bf16x2 __attribute__((ext_vector_type(2)));
typedef unsigned short mx_u16x2 __attribute__((ext_vector_type(2)));
typedef float mx_f32x2 __attribute__((ext_vector_type(2)));

FP4_D uint32_t mx_pk_max_u16(uint32_t a, uint32_t b) {
  union { uint32_t u; mx_u16x2 v; } x, y;
  x.u = a;
  y.u = b;
  x.v = __builtin_elementwise_max(x.v, y.v);
  return x.u;
}
FP4_D mx_bf16x2 mx_as_bf16x2(uint32_t u) {
  union { uint32_t u; mx_bf16x2 v; } c;
  c.u = u;
  return c.v;
}
FP4_D uint32_t mx_bits(mx_bf16x2 v) {
  union { mx_bf16x2 v; uint32_t u; } c;
  c.v = v;
  return c.u;
}
// The scaled converts divide by the scale (a power of two: exactly) and round to nearest, ties to the even code, saturating, in one step;
// checked on every bf16 pattern at seven scales and on a million fp32 values about the midpoints.
// Pairs of elements 2 I and 2 I + 1 of a word of eight codes; the second codes of 8 bits go to l.
template <int BITS, int I>
FP4_D void mx_pair(float a, float b, float s, uint32_t& h, uint32_t& l) {
  h = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(h, a, b, s, I);
  if constexpr (BITS == 8) {
    const mx_f32x2 d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(h, 1.0f, I);
    l = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(l, fmaf(-d.x, s, a), fmaf(-d.y, s, b), 0.125f * s, I);   // exact also where s h overflows
  }
}
template <int BITS, int I>
FP4_D void mx_pair(uint32_t ab, float s, uint32_t& h, uint32_t& l) {   // two bf16
  h = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(h, mx_as_bf16x2(ab), s, I);
  if constexpr (BITS == 8) {
    const mx_f32x2 d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(h, 1.0f, I);
    l = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(l, fmaf(-d.x, s, u2f(ab << 16)), fmaf(-d.y, s, u2f(ab & 0xffff0000u)), 0.125f * s, I);
  }
}
template <int BITS>
FP4_D void mx_encode8(const float* v, float s, uint32_t& h, uint32_t& l) {
  h = l = 0;
  mx_pair<BITS, 0>(v[0], v[1], s, h, l);
  mx_pair<BITS, 1>(v[2], v[3], s, h, l);
  mx_pair<BITS, 2>(v[4], v[5], s, h, l);
  mx_pair<BITS, 3>(v[6], v[7], s, h, l);
}
template <int BITS>
FP4_D void mx_encode8(const u32x4& w, float s, uint32_t& h, uint32_t& l) {   // eight bf16
  h = l = 0;
  mx_pair<BITS, 0>(w.x, s, h, l);
  mx_pair<BITS, 1>(w.y, s, h, l);
  mx_pair<BITS, 2>(w.z, s, h, l);
  mx_pair<BITS, 3>(w.w, s, h, l);
}
// The scale as the converts want it.  (For byte 255 the codes do not matter.)
FP4_D float mx_scale_f32(uint32_t byte) { return u2f(byte << 23); }
#endif  // __HIPCC__
