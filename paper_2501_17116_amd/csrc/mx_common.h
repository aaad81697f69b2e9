// Microscaled (MX) operands: blocks of 32 elements along the contraction share one power of two (E8M0, a byte: exponent + 127).
//
// An element is one E2M1 code h, x ~ s h (4 bits), or two, x ~ s (h + l / 8) (8 bits): h the nearest code to x / s, l the nearest to
// what is left at an eighth of the scale.  8 bits are two codes and not one E4M3 code because the matrix cores lose bits of 8-bit
// products: beside a large product of the same instruction the small ones are cut off at 2^-13 or so of it (measured, normal data: 5e-6
// of the result with one E4M3 operand, 1.5e-5 with two), while products of E2M1 codes come out exactly; two 4-bit instructions take as
// long as one 8-bit one; and their grid keeps more of the values: 37.5 dB on normal data (E4M3: 31.5), 34.8 on Student-t with three
// degrees of freedom.  In units of s it has every sixteenth up to 2 1/4; beyond, sixteenths within a quarter of a code, eighths further from
// one, and between 4 and 6 and above 6 quarters as well, with one gap of a half from 4 3/4 to 5 1/4; 6 3/4 is its largest value.
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
template <int BITS>
FP4_D void mx_encode8(const u32x4& a, const u32x4& b, float s, uint32_t& h, uint32_t& l) {   // eight fp32
  const float v[8] = {u2f(a.x), u2f(a.y), u2f(a.z), u2f(a.w), u2f(b.x), u2f(b.y), u2f(b.z), u2f(b.w)};
  mx_encode8<BITS>(v, s, h, l);
}
// The scale as the converts want it.  (For byte 255 the codes do not matter.)
FP4_D float mx_scale_f32(uint32_t byte) { return u2f(byte << 23); }
// max over a group of four lanes
FP4_D uint32_t mx_quad_max(uint32_t v) {
  uint32_t o = (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0xB1, 0xf, 0xf, true);   // lane ^ 1
  v = v > o ? v : o;
  o = (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x4E, 0xf, 0xf, true);            // lane ^ 2
  return v > o ? v : o;
}
// A 16-byte piece of a row: eight bf16 or four fp32 from column c on; zeros behind the row's end and in rows that are not there.  Without a
// branch, which would have each request waited for before the next: what is not there is read from where something is, and cleared.  ragged:
// whether rows end inside a piece (then element by element); the matrix has a row and a column.
template <class T>
FP4_D u32x4 mx_load_piece(const void* x, int64_t row, int64_t rows, int64_t cols, int64_t ld, int64_t c, bool ragged) {
  constexpr int N = 16 / sizeof(T);
  const T* const p = reinterpret_cast<const T*>(x) + min(row, rows - 1) * ld;
  u32x4 w;
  if (ragged) {
    uint32_t e[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const T v = p[min(c + i, cols - 1)];
      uint32_t bits;
      if constexpr (sizeof(T) == 2) bits = v;
      else bits = f2u(v);
      e[i] = row < rows && c + i < cols ? bits : 0u;
    }
    if constexpr (sizeof(T) == 2) w = u32x4{e[0] | e[1] << 16, e[2] | e[3] << 16, e[N - 4] | e[N - 3] << 16, e[N - 2] | e[N - 1] << 16};
    else w = u32x4{e[0], e[1], e[2], e[3]};
  } else {
    w = *reinterpret_cast<const u32x4*>(p + min(c, cols - N));
    const uint32_t in = row < rows && c < cols ? 0xffffffffu : 0u;
    w = u32x4{w.x & in, w.y & in, w.z & in, w.w & in};
  }
  return w;
}

FP4_D u32x4 mx_magnitudes_bf16(const u32x4& w) { return u32x4{w.x & 0x7fff7fffu, w.y & 0x7fff7fffu, w.z & 0x7fff7fffu, w.w & 0x7fff7fffu}; }
FP4_D uint32_t mx_amax_bf16(const u32x4& w) {   // bits of the largest magnitude of eight bf16, as fp32
  const u32x4 m = mx_magnitudes_bf16(w);
  const uint32_t a = mx_pk_max_u16(mx_pk_max_u16(m.x, m.y), mx_pk_max_u16(m.z, m.w));
  const uint32_t lo = a & 0xffffu, hi = a >> 16;
  return (lo > hi ? lo : hi) << 16;
}
FP4_D uint32_t mx_amax_f32(const u32x4& w) {
  const uint32_t a = w.x & 0x7fffffffu, b = w.y & 0x7fffffffu, c = w.z & 0x7fffffffu, d = w.w & 0x7fffffffu;
  const uint32_t ab = a > b ? a : b, cd = c > d ? c : d;
  return ab > cd ? ab : cd;
}

FP4_D uint32_t mx_pack_bf16x2(float a, float b) {
  mx_f32x2 f = {a, b};
  return mx_bits(__builtin_convertvector(f, mx_bf16x2));
}
// Four columns of a row, `left` of them there, with the addend where there is one.
template <bool OUT_BF16>
FP4_D void mx_store4(void* out, const float* addend, int64_t at, int64_t left, float (&y)[4]) {
  if (left >= 4) {
    if (addend) {
      const f32x4 a = *reinterpret_cast<const f32x4*>(addend + at);
      y[0] += a.x; y[1] += a.y; y[2] += a.z; y[3] += a.w;
    }
    if constexpr (OUT_BF16) *reinterpret_cast<u32x2*>(reinterpret_cast<uint16_t*>(out) + at) = u32x2{mx_pack_bf16x2(y[0], y[1]), mx_pack_bf16x2(y[2], y[3])};
    else *reinterpret_cast<f32x4*>(reinterpret_cast<float*>(out) + at) = f32x4{y[0], y[1], y[2], y[3]};
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (e < left) {
        const float v = addend ? y[e] + addend[at + e] : y[e];
        if constexpr (OUT_BF16) reinterpret_cast<uint16_t*>(out)[at + e] = (uint16_t)mx_pack_bf16x2(v, v);
        else reinterpret_cast<float*>(out)[at + e] = v;
      }
  }
}
#endif  // __HIPCC__
