// Product of two microscaled operands on the gfx950 F8F6F4 matrix cores, which take the blocks' scales themselves:
//
//   out[p, q] = sum over blocks b of 2^(eL[p, b] + eR[q, b]) * sum over k in b of vL[p, k] vR[q, k]   (+ addend[p, q])
//
// Both operands lie along the contraction (an "NT" product), each in 4 or 8 bits.  An operand of 8 bits is two planes of 4-bit codes, the
// second under an eighth of the scales, and the product is the sum of the planes' products: one, two or four passes over the contraction
// that add to the same accumulators.  Products of E2M1 codes are exact in the matrix core; sums are fp32; the one rounding to a narrower
// output type is the store's.
//
// v_mfma_scale_f32_32x32x64_f8f6f4, operand layout (found with one-hot operands): lane (l32, h) holds elements 32 h .. 32 h + 31 of row
// l32, sixteen bytes, and brings their scale, in the byte of its scale register that the instruction names.  A scale byte of 255 makes
// the row NaN, also over zero codes.
#include "mx_common.h"

#include <algorithm>

typedef int mx_i32x8 __attribute__((ext_vector_type(8)));
typedef float mx_f32x16 __attribute__((ext_vector_type(16)));

namespace {

struct MxGemm {
  const uint8_t *L, *R, *sL, *sR;
  const float* addend;
  void* out;
  int64_t P, Q, ldo;
  int64_t planeL, planeR;   // bytes of a plane of codes
  int64_t pitch;            // elements of a line
  int nl, nr;               // planes
};

// first operand: columns (Rt), second: rows (L); S: the byte of the scale registers, 0 or 2
template <int S>
FP4_D mx_f32x16 mx_mfma(const u32x4& r, const u32x4& l, const mx_f32x16& c, uint32_t sr, uint32_t sl) {
  const mx_i32x8 a = {(int)r.x, (int)r.y, (int)r.z, (int)r.w, 0, 0, 0, 0}, b = {(int)l.x, (int)l.y, (int)l.z, (int)l.w, 0, 0, 0, 0};
  if constexpr (S == 0) return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a, b, c, 4, 4, 0, (int)sr, 0, (int)sl);
  else return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a, b, c, 4, 4, 2, (int)sr, 2, (int)sl);
}

FP4_D uint32_t mx_pack_bf16x2(float a, float b) {
  mx_f32x2 f = {a, b};
  return mx_bits(__builtin_convertvector(f, mx_bf16x2));
}

// Four columns of a row; the row may end among them.
template <bool OUT_BF16>
FP4_D void mx_store4(const MxGemm& g, int64_t p, int64_t q, float (&y)[4]) {
  const int64_t at = p * g.ldo + q;
  if (q + 4 <= g.Q) {
    if (g.addend) {
      const f32x4 a = *reinterpret_cast<const f32x4*>(g.addend + at);
      y[0] += a.x; y[1] += a.y; y[2] += a.z; y[3] += a.w;
    }
    if constexpr (OUT_BF16) *reinterpret_cast<u32x2*>(reinterpret_cast<uint16_t*>(g.out) + at) = u32x2{mx_pack_bf16x2(y[0], y[1]), mx_pack_bf16x2(y[2], y[3])};
    else *reinterpret_cast<f32x4*>(reinterpret_cast<float*>(g.out) + at) = f32x4{y[0], y[1], y[2], y[3]};
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (q + e < g.Q) {
        const float v = g.addend ? y[e] + g.addend[at + e] : y[e];
        if constexpr (OUT_BF16) reinterpret_cast<uint16_t*>(g.out)[at + e] = (uint16_t)mx_pack_bf16x2(v, v);
        else reinterpret_cast<float*>(g.out)[at + e] = v;
      }
  }
}

// 64 x 64 outputs a workgroup, 32 x 32 a wave, operands straight from memory to the matrix core's registers, 512 codes of the contraction a
// step.  Rows past the matrix's edge repeat its last one and are not stored.
template <bool OUT_BF16>
__global__ __launch_bounds__(256) void mx_gemm_small_kernel(MxGemm g) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int l32 = lane & 31, h = lane >> 5;
  const int64_t P0 = (int64_t)blockIdx.x * 64 + (wave & 1) * 32, Q0 = (int64_t)blockIdx.y * 64 + (wave >> 1) * 32;
  const int64_t p = std::min(P0 + l32, g.P - 1), q = std::min(Q0 + l32, g.Q - 1);
  const uint32_t *sl = reinterpret_cast<const uint32_t*>(g.sL + p * (g.pitch / MX_BLOCK)), *sr = reinterpret_cast<const uint32_t*>(g.sR + q * (g.pitch / MX_BLOCK));
  mx_f32x16 acc;
#pragma unroll
  for (int v = 0; v < 16; ++v) acc[v] = 0.0f;
  for (int pass = 0; pass < g.nl * g.nr; ++pass) {
    const int pl = pass % g.nl, pr = pass / g.nl;
    const uint8_t *l = g.L + pl * g.planeL + p * (g.pitch / 2) + h * 16, *r = g.R + pr * g.planeR + q * (g.pitch / 2) + h * 16;
    const uint32_t lessl = pl ? MX_EIGHTH : 0u, lessr = pr ? MX_EIGHTH : 0u;
    for (int64_t k = 0; k < g.pitch / 128; k += 4) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {   // 128 codes, one word of scales
        const uint32_t bl = (sl[k + j] - lessl) >> (8 * h), br = (sr[k + j] - lessr) >> (8 * h);
        const u32x4 *lv = reinterpret_cast<const u32x4*>(l + (k + j) * 64), *rv = reinterpret_cast<const u32x4*>(r + (k + j) * 64);
        acc = mx_mfma<0>(rv[0], lv[0], acc, br, bl);
        acc = mx_mfma<2>(rv[2], lv[2], acc, br, bl);
      }
    }
  }
  if (P0 + l32 >= g.P) return;
#pragma unroll
  for (int b = 0; b < 4; ++b) {
    const int64_t qc = Q0 + b * 8 + h * 4;
    float y[4] = {acc[b * 4], acc[b * 4 + 1], acc[b * 4 + 2], acc[b * 4 + 3]};
    if (qc < g.Q) mx_store4<OUT_BF16>(g, P0 + l32, qc, y);
  }
}

template <bool OUT_BF16>
int launch(const MxGemm& g, hipStream_t s) {
  const dim3 grid((unsigned)((g.P + 63) / 64), (unsigned)((g.Q + 63) / 64));
  hipLaunchKernelGGL((mx_gemm_small_kernel<OUT_BF16>), grid, dim3(256), 0, s, g);
  FP4_CHECK_LAUNCH();
  return FP4_OK;
}

}  // namespace

// P and Q are at least 1; Kc may be 0.
int mx_launch_gemm(const uint8_t* L, const uint8_t* sL, int bits_l, const uint8_t* R, const uint8_t* sR, int bits_r, int64_t P, int64_t Q, int64_t Kc,
                   const float* addend, void* out, int out_bf16, int64_t ldo, hipStream_t s) {
  MxGemm g;
  g.L = L; g.R = R; g.sL = sL; g.sR = sR;
  g.addend = addend;
  g.out = out;
  g.P = P; g.Q = Q; g.ldo = ldo;
  g.pitch = mx_pitch_of(Kc);
  g.planeL = P * (g.pitch / 2);
  g.planeR = Q * (g.pitch / 2);
  g.nl = bits_l / 4;
  g.nr = bits_r / 4;
  return out_bf16 ? launch<true>(g, s) : launch<false>(g, s);
}
