// What stays in high precision: elements in bf16 or fp32, arithmetic and sums in fp32.
#pragma once
#include "fp4_common.h"

constexpr int64_t HP_MAX_DIM = int64_t{1} << 21;   // of any dimension: keeps every grid and every tile's byte offsets within 32 bits
constexpr int64_t HP_NORM_MAX_D = 16384;           // a row is held in one workgroup's registers

#if defined(__HIPCC__)
typedef __bf16 hp_bf16x2 __attribute__((ext_vector_type(2)));
typedef float hp_f32x2 __attribute__((ext_vector_type(2)));

FP4_D uint32_t hp_pack_bf16(float a, float b) {   // to nearest, ties to even
  const hp_f32x2 f = {a, b};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f, hp_bf16x2));
}

// Eight elements as they lie in memory.
template <class T> struct Raw8;
template <> struct Raw8<BF16> {
  u32x4 w;
  FP4_D void zero() { w = u32x4{0, 0, 0, 0}; }
  FP4_D float get(int i) const { return u2f(i & 1 ? w[i >> 1] & 0xffff0000u : w[i >> 1] << 16); }
};
template <> struct Raw8<F32> {
  f32x4 a, b;
  FP4_D void zero() { a = b = f32x4{0, 0, 0, 0}; }
  FP4_D float get(int i) const { return i < 4 ? a[i & 3] : b[i & 3]; }
};

// Elements c .. c + 7 of a row (its start 16-byte aligned, c a multiple of 8) that ends at `cols`; zeros behind its end.
FP4_D Raw8<BF16> hp_load8(const BF16*, const void* row, int64_t c, int64_t cols) {
  Raw8<BF16> r;
  const uint16_t* p = reinterpret_cast<const uint16_t*>(row) + c;
  if (c + 8 <= cols) {
    r.w = *reinterpret_cast<const u32x4*>(p);
  } else {
    uint32_t e[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) e[i] = c + i < cols ? p[i] : 0u;
    r.w = u32x4{e[0] | e[1] << 16, e[2] | e[3] << 16, e[4] | e[5] << 16, e[6] | e[7] << 16};
  }
  return r;
}
FP4_D Raw8<F32> hp_load8(const F32*, const void* row, int64_t c, int64_t cols) {
  Raw8<F32> r;
  const float* p = reinterpret_cast<const float*>(row) + c;
  if (c + 8 <= cols) {
    r.a = *reinterpret_cast<const f32x4*>(p);
    r.b = *reinterpret_cast<const f32x4*>(p + 4);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      r.a[i] = c + i < cols ? p[i] : 0.0f;
      r.b[i] = c + 4 + i < cols ? p[4 + i] : 0.0f;
    }
  }
  return r;
}
template <class T>
FP4_D Raw8<T> hp_load8(const void* row, int64_t c, int64_t cols) { return hp_load8((const T*)nullptr, row, c, cols); }

FP4_D void hp_store8(const BF16*, void* row, int64_t c, int64_t cols, const float (&v)[8]) {
  uint16_t* p = reinterpret_cast<uint16_t*>(row) + c;
  const u32x4 w = {hp_pack_bf16(v[0], v[1]), hp_pack_bf16(v[2], v[3]), hp_pack_bf16(v[4], v[5]), hp_pack_bf16(v[6], v[7])};
  if (c + 8 <= cols) {
    *reinterpret_cast<u32x4*>(p) = w;
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (c + i < cols) p[i] = (uint16_t)(w[i >> 1] >> (i & 1) * 16);
  }
}
FP4_D void hp_store8(const F32*, void* row, int64_t c, int64_t cols, const float (&v)[8]) {
  float* p = reinterpret_cast<float*>(row) + c;
  if (c + 8 <= cols) {
    *reinterpret_cast<f32x4*>(p) = f32x4{v[0], v[1], v[2], v[3]};
    *reinterpret_cast<f32x4*>(p + 4) = f32x4{v[4], v[5], v[6], v[7]};
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (c + i < cols) p[i] = v[i];
  }
}
template <class T>
FP4_D void hp_store8(void* row, int64_t c, int64_t cols, const float (&v)[8]) { hp_store8((const T*)nullptr, row, c, cols, v); }

template <class T> struct HpSize;
template <> struct HpSize<BF16> { static constexpr int value = 2; };
template <> struct HpSize<F32> { static constexpr int value = 4; };
template <class T>
FP4_D const uint8_t* hp_row(const void* x, int64_t row, int64_t ld) { return reinterpret_cast<const uint8_t*>(x) + row * ld * HpSize<T>::value; }
template <class T>
FP4_D uint8_t* hp_row(void* x, int64_t row, int64_t ld) { return reinterpret_cast<uint8_t*>(x) + row * ld * HpSize<T>::value; }

FP4_D float hp_wave_sum(float v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
  return v;
}
#endif  // __HIPCC__
