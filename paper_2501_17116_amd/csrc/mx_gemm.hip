// Product of two microscaled operands on the gfx950 F8F6F4 matrix cores, which take the blocks' scales themselves:
//
//   out[p, q] = sum over blocks b of 2^(eL[p, b] + eR[q, b]) * sum over k in b of vL[p, k] vR[q, k]   (+ addend[p, q])
//
// Both operands lie along the contraction (an "NT" product), each in 4 or 8 bits.  An operand of 8 bits is two planes of 4-bit codes, the
// second under an eighth of the scales, and the product is the sum of the planes' products: one, two or four passes over the contraction
// that add to the same accumulators.  Products of E2M1 codes are exact in the matrix core; sums are fp32; the one rounding to a narrower
// output type is the store's.
//
// Sizes in this file are P x Q x contraction, outputs first.
//
// v_mfma_scale_f32_32x32x64_f8f6f4, operand layout (found with one-hot operands): lane (l32, h) holds elements 32 h .. 32 h + 31 of row
// l32, sixteen bytes, and brings their scale, in the byte of its scale register that the instruction names.  A scale byte of 255 makes
// the row NaN, also over zero codes.
#include "mx_common.h"
#include "mx_tiling.h"
#include "fp4_measure.h"

#include <algorithm>
#include <type_traits>
#include <utility>

typedef int mx_i32x8 __attribute__((ext_vector_type(8)));
typedef float mx_f32x16 __attribute__((ext_vector_type(16)));

int fp4_compute_units_of_current_device();
int mx_check_gemm(const fp4_mx* l, const fp4_mx* rt, const float* addend, const void* out, int out_dt, int64_t ldo);
int mx_launch_few(const uint8_t* L, const uint8_t* sL, const void* x, int x_bf16, int64_t ldx, int bits_l, const uint8_t* R, const uint8_t* sR, int bits_r,
                  int64_t P, int64_t Q, int64_t Kc, const float* addend, void* out, int out_bf16, int64_t ldo, hipStream_t s);

namespace {

struct MxGemm {
  const uint8_t *L, *R, *sL, *sR;
  const float* addend;
  void* out;
  int64_t P, Q, ldo;
  int64_t planeL, planeR;   // bytes of a plane of codes
  int64_t pitch;            // elements of a line
  int steps;                // of 256 codes a pass
  int nl, nr;               // planes
  int tiles_p, tiles_q;
  int first, count;         // tiles of this launch, in the order of tile_at
  bool stream;              // the output passes the caches by
};

template <class F, int... I>
FP4_D void static_for_impl(F&& f, std::integer_sequence<int, I...>) {
  (f(std::integral_constant<int, I>{}), ...);
}
template <int N, class F>
FP4_D void static_for(F&& f) {
  static_for_impl(f, std::make_integer_sequence<int, N>{});
}

// First operand: columns (Rt), second: rows (L).  S: the byte of the scale registers.  A step is 256 codes of a line, of which lane
// half h takes 128 h .. 128 h + 127: its four words of codes a slice, its one word of scales the four slices in order, so that no scale
// has to be moved to its place (the instruction does not mind which elements of a line meet, only that those of both operands do).
template <int S>
FP4_D mx_f32x16 mx_mfma(const u32x4& r, const u32x4& l, const mx_f32x16& c, uint32_t sr, uint32_t sl) {
  const mx_i32x8 a = {(int)r.x, (int)r.y, (int)r.z, (int)r.w, 0, 0, 0, 0}, b = {(int)l.x, (int)l.y, (int)l.z, (int)l.w, 0, 0, 0, 0};
  if constexpr (S == 0) return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a, b, c, 4, 4, 0, (int)sr, 0, (int)sl);
  else if constexpr (S == 1) return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a, b, c, 4, 4, 1, (int)sr, 1, (int)sl);
  else if constexpr (S == 2) return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a, b, c, 4, 4, 2, (int)sr, 2, (int)sl);
  else return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a, b, c, 4, 4, 3, (int)sr, 3, (int)sl);
}

// 64 x 64 outputs a workgroup, 32 x 32 a wave, operands straight from memory to the matrix core's registers.  Rows past the matrix's edge
// repeat its last one and are not stored.  For short contractions, where a start through LDS costs more than it saves: one round trip to
// memory a step is what bounds it (249 x 2400 over 264 5.3 us, a launch by itself 3.4).
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
    const uint8_t *l = g.L + pl * g.planeL + p * (g.pitch / 2) + h * 64, *r = g.R + pr * g.planeR + q * (g.pitch / 2) + h * 64;
    const uint32_t lessl = pl ? MX_EIGHTH : 0u, lessr = pr ? MX_EIGHTH : 0u;
    for (int k = 0; k < g.steps; ++k) {   // 256 codes, one word of scales
      const uint32_t bl = sl[2 * k + h] - lessl, br = sr[2 * k + h] - lessr;
      const u32x4 *lv = reinterpret_cast<const u32x4*>(l + k * 128), *rv = reinterpret_cast<const u32x4*>(r + k * 128);
      static_for<4>([&](auto sc) {
        constexpr int s = decltype(sc)::value;
        acc = mx_mfma<s>(rv[s], lv[s], acc, br, bl);
      });
    }
  }
  if (P0 + l32 >= g.P) return;
#pragma unroll
  for (int b = 0; b < 4; ++b) {
    const int64_t qc = Q0 + b * 8 + h * 4;
    float y[4] = {acc[b * 4], acc[b * 4 + 1], acc[b * 4 + 2], acc[b * 4 + 3]};
    if (qc < g.Q) mx_store4<OUT_BF16>(g.out, g.addend, (P0 + l32) * g.ldo + qc, g.Q - qc, y);
  }
}

// ---- 256 x 256, 256 x 192 -------------------------------------------------------------------------------------------------------
// For outputs that go round the chip in such tiles.  Eight waves, PJ x QI blocks of 32 x 32 each (256 columns: 2 along rows x 4 along columns,
// 128 x 64 each; 192: 4 x 2, 64 x 96 each), persistent workgroups, K step 256 codes.  Operands come into two LDS stages by direct-to-LDS
// loads, the scales of two steps at a time (16 bytes of every row, one load a thread) into a ring of two of their own; the two waves of a
// SIMD alternate between a compute phase (the matrix instructions of two slices) and a memory phase (the fragments of the next two
// slices, and once a step its share of the loads of the step after next), half a period apart.  Sums leave from their registers, so that the
// next tile's first two steps travel during the stores.
// An operand stage: row r takes bytes [128 r, 128 r + 128), its 16-byte chunk c sits in slot c ^ ((r >> 1) & 7), so that sixteen rows
// reading one chunk touch sixteen different bank groups.
// Measured (4 x 4 bits, bf16 out, repeated calls): 8192 x 2048 x 5504 48 us, 8192 x 11008 x 4096 203 us, 16384 x 12288 x 4096 419 us (3.7 - 3.9e15
// operations/s); 8 x 4 bits, 4096 x 4096 x 8192 127 us (4.3e15 of codes).  The issue loop alone over random operands reaches 6.4e15.  Bound:
// the matrix cores and power: over 16384 x 12288 x 4096 the clock falls to 1.8 - 1.9 GHz, and of its cycles the matrix cores are busy in
// 49 %, LDS in 29 % (a quarter of that in conflicts).  Without its loads the same loop reaches 5.5e15, with loads that hit L2 4.6e15; misses and
// the stores' share of memory are the rest.
// Tried: half steps of 64 bytes of a row with three on their way (1.5 steps ahead instead of one): 5 % faster at the largest outputs, 5 %
// slower elsewhere, as twice the rows a
// load cost more than the distance gave.  Parking the sums in LDS for stores of 128 bytes instead of the swaps' 64: 50.0 against 48.4,
// 220 against 210 us.
constexpr int BP = 256, BKB = 128;
constexpr int BWAVES = 8;
template <int BQ> struct BigShape {
  static constexpr int WP = BQ == 256 ? 2 : 4;                   // waves along rows
  static constexpr int PJ = BP / 32 / WP, QI = BQ / 32 / (BWAVES / WP);
  static constexpr int LDL = BP * 8 / (BWAVES * 64), LDR = BQ * 8 / (BWAVES * 64);   // 16-byte chunks a thread and step
  static constexpr int OP_L = BP * BKB, STAGE = (BP + BQ) * BKB;
  static constexpr int SC_BASE = 2 * STAGE, SC = 2 * 256 * 16;
  static constexpr int SMEM = SC_BASE + 2 * SC;
  static_assert(SMEM <= 160 * 1024, "LDS budget");
};
// Tile rows side by side: the 32 CUs of an XCD work on 4 x 8 tiles, whose rows' operand stays in its L2 while the columns' passes (16384 x 12288
// x 4096 with 4 / 6 / 8 / 16 of them 419 / 422 / 430 / 435 us, 4096 x 11008 x 8192 in 8 x 4 bits 387 / 385 / 391 / 405).
constexpr int GROUP_P = 4;
constexpr uint32_t PAST_THE_END = 0xf0000000u;   // behind any descriptor: arrives as zeros, is not stored
constexpr int64_t WIDE_LDO = 1 << 24;            // 32 rows of so many floats stay below PAST_THE_END

FP4_D void tile_at(const MxGemm& g, int id, int& tp, int& tq) {
  const int in_group = GROUP_P * g.tiles_q, group = id / in_group, first_p = group * GROUP_P;
  const int gsz = min(g.tiles_p - first_p, GROUP_P);
  tp = first_p + (id % in_group) % gsz;
  tq = (id % in_group) / gsz;
}

FP4_D const uint8_t* uniform_ptr(const uint8_t* p) {
  const uint64_t v = (uint64_t)p;
  const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)v), hi = __builtin_amdgcn_readfirstlane((uint32_t)(v >> 32));
  return (const uint8_t*)(((uint64_t)hi << 32) | lo);
}
FP4_D __amdgpu_buffer_rsrc_t rows_rsrc(const uint8_t* p, int64_t rows, int64_t pitch) {   // over so many rows; they stay below 2^30 bytes
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(uniform_ptr(p)), 0, __builtin_amdgcn_readfirstlane((int)(rows * pitch)), 0x00020000);
}
// global -> LDS without passing through registers, a wave's lanes one behind another from `lds` on.  (Functions of their own and no templates:
// with arguments that depend on a template parameter the builtin makes the compiler drop the kernel's host stub.)
FP4_D void to_lds16(__amdgpu_buffer_rsrc_t rsrc, uint8_t* lds, uint32_t voff, int soff) {
  __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (__attribute__((address_space(3))) void*)lds, 16, voff, soff, 0, 0);
}
FP4_D void to_lds4(__amdgpu_buffer_rsrc_t rsrc, uint8_t* lds, uint32_t voff, int soff) {
  __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (__attribute__((address_space(3))) void*)lds, 4, voff, soff, 0, 0);
}

// Until all but the latest N requests of this wave have landed, and (READS) its reads of LDS are over.
template <int N, bool READS = false>
FP4_D void wait_loads() {
  static_assert(N < 64, "what the counter holds");
  __builtin_amdgcn_s_waitcnt((READS ? 0x0070 : 0x0f70) | (N & 15) | ((N >> 4) << 14));
}

// STREAM: past the caches
template <bool STREAM>
FP4_D void store16(__amdgpu_buffer_rsrc_t rsrc, const u32x4& x, uint32_t voff) {
  __builtin_amdgcn_raw_buffer_store_b128(x, rsrc, voff, 0, STREAM ? 18 : 0);
}
FP4_D void store8(__amdgpu_buffer_rsrc_t rsrc, const u32x2& x, uint32_t voff) { __builtin_amdgcn_raw_buffer_store_b64(x, rsrc, voff, 0, 0); }
FP4_D f32x4 load16(__amdgpu_buffer_rsrc_t rsrc, uint32_t voff) { return __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(rsrc, voff, 0, 0)); }

// Between the lanes' four groups of sixteen: the second and fourth group of a with the first and third of b; the upper two groups of a
// with the lower two of b.
FP4_D void swap16(uint32_t& a, uint32_t& b) {
  const auto r = __builtin_amdgcn_permlane16_swap(a, b, false, false);
  a = r[0]; b = r[1];
}
FP4_D void swap16(float& a, float& b) {
  uint32_t x = __builtin_bit_cast(uint32_t, a), y = __builtin_bit_cast(uint32_t, b);
  swap16(x, y);
  a = __builtin_bit_cast(float, x);
  b = __builtin_bit_cast(float, y);
}
FP4_D void swap32(uint32_t& a, uint32_t& b) {
  const auto r = __builtin_amdgcn_permlane32_swap(a, b, false, false);
  a = r[0]; b = r[1];
}

// Eight columns of a row from q on, y without the addend.
template <bool OUT_BF16>
FP4_D void store8(const MxGemm& g, int64_t at, int64_t left, const float (&y)[8]) {
  if (left >= 8) {
    if constexpr (OUT_BF16) {
      *reinterpret_cast<u32x4*>(reinterpret_cast<uint16_t*>(g.out) + at) =
          u32x4{mx_pack_bf16x2(y[0], y[1]), mx_pack_bf16x2(y[2], y[3]), mx_pack_bf16x2(y[4], y[5]), mx_pack_bf16x2(y[6], y[7])};
    } else {
      float* o = reinterpret_cast<float*>(g.out) + at;
      *reinterpret_cast<f32x4*>(o) = f32x4{y[0], y[1], y[2], y[3]};
      *reinterpret_cast<f32x4*>(o + 4) = f32x4{y[4], y[5], y[6], y[7]};
    }
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e < left) {
        if constexpr (OUT_BF16) reinterpret_cast<uint16_t*>(g.out)[at + e] = (uint16_t)mx_pack_bf16x2(y[e], y[e]);
        else reinterpret_cast<float*>(g.out)[at + e] = y[e];
      }
  }
}
FP4_D void load_addend8(const MxGemm& g, int64_t at, int64_t left, float (&a)[8]) {
  if (left >= 8) {
    const f32x4 u = *reinterpret_cast<const f32x4*>(g.addend + at), v = *reinterpret_cast<const f32x4*>(g.addend + at + 4);
    a[0] = u.x; a[1] = u.y; a[2] = u.z; a[3] = u.w;
    a[4] = v.x; a[5] = v.y; a[6] = v.z; a[7] = v.w;
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) a[e] = e < left ? g.addend[at + e] : 0.0f;
  }
}

template <int BQ, bool OUT_BF16>
__global__ __launch_bounds__(BWAVES * 64) void mx_gemm_big_kernel(MxGemm g) {
  using S = BigShape<BQ>;
  constexpr int PJ = S::PJ, QI = S::QI;
  __shared__ __attribute__((aligned(16))) uint8_t smem[S::SMEM];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wave_p = wave % S::WP, wave_q = wave / S::WP;
  const int l32 = lane & 31, h = lane >> 5;
  // each XCD a contiguous run of tiles, so that those that share rows meet in one L2
  const int per_xcd = (g.count + 7) / 8;
  const int xcd = (int)(blockIdx.x % 8), stride = (int)(gridDim.x / 8);
  const int run_end = min(g.count, (xcd + 1) * per_xcd);
  int lid = xcd * per_xcd + (int)(blockIdx.x / 8);
  if (lid >= run_end) return;

  const int64_t rowb = g.pitch / 2, rows_s = g.pitch / MX_BLOCK;
  const int KT = (int)(g.pitch / 256), T = KT * g.nl * g.nr;   // steps of a pass (even), of all passes
  int64_t P0 = 0, Q0 = 0;
  __amdgpu_buffer_rsrc_t rsrcL, rsrcR, rsrcS;
  uint32_t offL[S::LDL], offR[S::LDR], offS;
  int ld_k = 0, ld_pass = 0, sc_k = 0;   // the step in its pass that is requested next, and the pair of steps whose scales are
  auto planes = [&](int pass) {
    rsrcL = rows_rsrc(g.L + (pass % g.nl) * g.planeL + P0 * rowb, min(g.P - P0, (int64_t)BP), rowb);
    rsrcR = rows_rsrc(g.R + (pass / g.nl) * g.planeR + Q0 * rowb, min(g.Q - Q0, (int64_t)BQ), rowb);
  };
  auto tile_scalars = [&](int id) {
    int tp, tq;
    tile_at(g, id, tp, tq);
    P0 = (int64_t)tp * BP;
    Q0 = (int64_t)tq * BQ;
    ld_k = ld_pass = sc_k = 0;
    planes(0);
    rsrcS = wave < 4 ? rows_rsrc(g.sL + P0 * rows_s, min(g.P - P0, (int64_t)BP), rows_s) : rows_rsrc(g.sR + Q0 * rows_s, min(g.Q - Q0, (int64_t)BQ), rows_s);
  };
  // rebuilt where they are needed from a copy of the lane id that the optimizer cannot see through: kept across the epilogue they
  // would cost registers there
  auto tile_offsets = [&]() {
    int ln = lane;
    asm volatile("" : "+v"(ln));
    auto offset = [&](int row, int64_t first, int64_t rows) {   // of a lane's chunk; rows past the edge re-read the last row
      return (uint32_t)((min(first + row, rows - 1) - first) * rowb + ((ln & 7) ^ ((row >> 1) & 7)) * 16);
    };
#pragma unroll
    for (int j = 0; j < S::LDL; ++j) offL[j] = offset(8 * (wave * S::LDL + j) + (ln >> 3), P0, g.P);
#pragma unroll
    for (int j = 0; j < S::LDR; ++j) offR[j] = offset(8 * (wave * S::LDR + j) + (ln >> 3), Q0, g.Q);
    const int row = (wave & 3) * 64 + ln;
    offS = (uint32_t)(wave < 4 ? (min(P0 + row, g.P - 1) - P0) * rows_s : (min(Q0 + row, g.Q - 1) - Q0) * rows_s);
  };
  auto load_step = [&](int buf) {
#pragma unroll
    for (int j = 0; j < S::LDL; ++j) {
      to_lds16(rsrcL, smem + buf * S::STAGE + (wave * S::LDL + j) * 1024, offL[j], ld_k * BKB);
      if (j < S::LDR) to_lds16(rsrcR, smem + buf * S::STAGE + S::OP_L + (wave * S::LDR + j) * 1024, offR[j < S::LDR ? j : 0], ld_k * BKB);
    }
    if (++ld_k == KT) {
      ld_k = 0;
      if (++ld_pass < g.nl * g.nr) planes(ld_pass);
    }
  };
  auto load_scales = [&](int buf) {   // wave w: rows 64 w .. of L, then of Rt (those behind a tile's 192 arrive as zeros)
    to_lds16(rsrcS, smem + S::SC_BASE + buf * S::SC + wave * 1024, offS, sc_k * 16);
    if (++sc_k == KT / 2) sc_k = 0;
  };

  // Fragments: lane (l32, h) takes chunk 4 h + slice of rows l32 + 32 j; the swizzle only depends on l32.
  const int key = (l32 >> 1) & 7;
  int frag_l[4], frag_r[4];
#pragma unroll
  for (int s = 0; s < 4; ++s) {
    frag_l[s] = (wave_p * (PJ * 32) + l32) * BKB + ((4 * h + s) ^ key) * 16;
    frag_r[s] = S::OP_L + (wave_q * (QI * 32) + l32) * BKB + ((4 * h + s) ^ key) * 16;
  }
  const int scale_l = S::SC_BASE + (wave_p * (PJ * 32) + l32) * 16 + h * 4, scale_r = S::SC_BASE + BP * 16 + (wave_q * (QI * 32) + l32) * 16 + h * 4;
  u32x4 fl[2][PJ], fr[2][QI];
  uint32_t sl[PJ], sr[QI], lessl = 0, lessr = 0;
  auto read_frags = [&](int buf, int half) {
#pragma unroll
    for (int s = 0; s < 2; ++s) {
#pragma unroll
      for (int j = 0; j < QI; ++j) fr[s][j] = *reinterpret_cast<const u32x4*>(smem + buf * S::STAGE + frag_r[2 * half + s] + j * 32 * BKB);
#pragma unroll
      for (int j = 0; j < PJ; ++j) fl[s][j] = *reinterpret_cast<const u32x4*>(smem + buf * S::STAGE + frag_l[2 * half + s] + j * 32 * BKB);
    }
  };
  auto read_scales = [&](int buf, int parity) {
#pragma unroll
    for (int j = 0; j < QI; ++j) sr[j] = *reinterpret_cast<const uint32_t*>(smem + buf * S::SC + scale_r + parity * 8 + j * 512) - lessr;
#pragma unroll
    for (int j = 0; j < PJ; ++j) sl[j] = *reinterpret_cast<const uint32_t*>(smem + buf * S::SC + scale_l + parity * 8 + j * 512) - lessl;
  };
  mx_f32x16 acc[QI][PJ];

  tile_scalars(lid);
  tile_offsets();
  const auto first_requests = [&]() {
    load_step(0);
    load_scales(0);
    load_step(1);
    load_scales(1);
  };
  first_requests();
  // Stores of the tile before that were issued after these requests and that no wait has to include: so many, or none that are known
  constexpr int STORES = PJ * QI * (OUT_BF16 ? 2 : 4);
  bool counted = false;
  while (true) {
    const int64_t eP0 = P0, eQ0 = Q0;   // of this tile, for its epilogue
    tile_offsets();
#pragma unroll
    for (int i = 0; i < QI; ++i)
#pragma unroll
      for (int j = 0; j < PJ; ++j)
#pragma unroll
        for (int v = 0; v < 16; ++v) acc[i][j][v] = 0.0f;
    constexpr int n = S::LDL + S::LDR + 1;   // all but the second step's
    if (counted) wait_loads<n + STORES>();
    else wait_loads<n>();
    __builtin_amdgcn_s_barrier();   // a bare one: the fence of __syncthreads() would wait for the second stage too
    asm volatile("" ::: "memory");
    lessl = lessr = 0;
    read_scales(0, 0);
    read_frags(0, 0);
    int rd_k = 0, rd_pass = 0;   // of the step whose scales are held
    const bool second_group = wave >= BWAVES / 2;
    if (second_group) __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    for (int t = 0; t < T; t += 2) {
      const int sbuf = (t >> 1) & 1;
      static_for<2>([&](auto ec) {
        constexpr int e = decltype(ec)::value;
        static_for<2>([&](auto hc) {
          constexpr int half = decltype(hc)::value;
          __builtin_amdgcn_sched_barrier(0);
          __builtin_amdgcn_s_setprio(1);
#pragma unroll
          for (int qi = 0; qi < QI; ++qi)
#pragma unroll
            for (int pj = 0; pj < PJ; ++pj) acc[qi][pj] = mx_mfma<2 * half>(fr[0][qi], fl[0][pj], acc[qi][pj], sr[qi], sl[pj]);
#pragma unroll
          for (int qi = 0; qi < QI; ++qi)
#pragma unroll
            for (int pj = 0; pj < PJ; ++pj) acc[qi][pj] = mx_mfma<2 * half + 1>(fr[1][qi], fl[1][pj], acc[qi][pj], sr[qi], sl[pj]);
#pragma unroll
          for (int qi = 0; qi < QI; ++qi)
#pragma unroll
            for (int pj = 0; pj < PJ; pj += 2) asm volatile("" : "+v"(acc[qi][pj]), "+v"(acc[qi][pj + 1]));
          __builtin_amdgcn_s_setprio(0);
          __builtin_amdgcn_sched_barrier(0);
          if constexpr (half == 1) {   // the next step is first read in this memory phase: its loads have landed by the barrier before
            if (!second_group) {
              if (e == 0 && t == 0 && counted) wait_loads<STORES>();
              else wait_loads<0>();
            }
          }
          __builtin_amdgcn_s_barrier();
          asm volatile("" ::: "memory");
          __builtin_amdgcn_sched_barrier(0);
          if constexpr (half == 0) {
            read_frags(e, 1);
            // its share of the next step has landed before the first group reads it, and these reads of a stage that the first group
            // fills next are over
            if (second_group) {
              if (e == 0 && t == 0 && counted) wait_loads<STORES, true>();
              else wait_loads<0, true>();
            }
          } else {
            if (++rd_k == KT) {
              rd_k = 0;
              ++rd_pass;
              lessl = rd_pass % g.nl ? MX_EIGHTH : 0u;
              lessr = rd_pass / g.nl ? MX_EIGHTH : 0u;
            }
            read_scales(e == 0 ? sbuf : sbuf ^ 1, e ^ 1);
            read_frags(e ^ 1, 0);
            if (t + e + 2 < T) load_step(e);
            if constexpr (e == 1) {
              if (t + 4 < T) load_scales(sbuf);
            }
          }
          __builtin_amdgcn_sched_barrier(0);
          __builtin_amdgcn_s_barrier();
          asm volatile("" ::: "memory");
        });
      });
    }
    if (!second_group) __builtin_amdgcn_s_barrier();
    __syncthreads();   // every wave is done with the stages

    const int next = lid + stride;
    const bool has_next = next < run_end;
    if (has_next) {
      tile_scalars(next);
      tile_offsets();
      first_requests();
    }
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);

    // Epilogue.  A lane holds four columns in a row of every eight of one row; swaps between the lanes' groups of sixteen give each store
    // 64 bytes of a row, without LDS, whose stages the next tile's first steps are already on their way to.
    int ln = lane;
    asm volatile("" : "+v"(ln));
    const int r16 = ln & 15, unit = (ln >> 5) + (ln >> 3 & 2);   // of a store: the row, and the piece of 16 bytes
    const int64_t q0 = eQ0 + wave_q * (QI * 32), left = g.Q - q0;
    counted = !(g.addend && OUT_BF16) && g.ldo <= WIDE_LDO && (g.Q % 8 == 0 || left >= QI * 32);
    constexpr int ES = OUT_BF16 ? 2 : 4;
    static_for<PJ>([&](auto pc) {
      constexpr int pj = decltype(pc)::value;
      const int64_t p0 = eP0 + (wave_p * PJ + pj) * 32, rows = max(min(g.P - p0, (int64_t)32), (int64_t)0);
      const uint32_t line = (uint32_t)g.ldo;
      // rows behind the edge are behind the descriptor, columns are sent there
      const auto at = [&](int row, int col, int size) { return col < left ? ((uint32_t)row * line + (uint32_t)col) * (uint32_t)size : PAST_THE_END; };
      const __amdgpu_buffer_rsrc_t rsrc = rows_rsrc((const uint8_t*)g.out + (p0 * g.ldo + q0) * ES, rows, g.ldo * ES);
      const auto put = [&](auto stream, const u32x4& x, uint32_t o) { store16<decltype(stream)::value>(rsrc, x, o); };
      const auto store_all = [&](auto stream) {
        if (OUT_BF16 && (decltype(stream)::value || counted)) {   // no addend
          static_for<QI>([&](auto qc) {
            constexpr int qi = decltype(qc)::value;
            const mx_f32x16& c = acc[qi][pj];
            uint32_t d[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) d[i] = mx_pack_bf16x2(c[2 * i], c[2 * i + 1]);
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              swap32(d[i], d[2 + i]);
              swap32(d[4 + i], d[6 + i]);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) swap16(d[i], d[4 + i]);
            put(stream, u32x4{d[0], d[1], d[2], d[3]}, at(r16, qi * 32 + unit * 8, 2));
            put(stream, u32x4{d[4], d[5], d[6], d[7]}, at(16 + r16, qi * 32 + unit * 8, 2));
          });
          return;
        }
        const bool wide = g.ldo > WIDE_LDO || (g.Q % 8 && left < QI * 32);
        f32x4 a[QI * 2][2] = {};
        if (g.addend && !wide) {   // all of it is requested before the first store: loads and stores count on one in-order counter
          const __amdgpu_buffer_rsrc_t from = rows_rsrc((const uint8_t*)(g.addend + p0 * g.ldo + q0), rows, g.ldo * 4);
#pragma unroll
          for (int j = 0; j < 2 * QI; ++j)
#pragma unroll
            for (int v = 0; v < 2; ++v) a[j][v] = load16(from, at(16 * v + r16, 16 * j + 4 * unit, 4));
        }
        static_for<QI * 2>([&](auto jc) {   // columns 16 j + 4 unit on, of the first sixteen rows and of the others
          constexpr int j = decltype(jc)::value;
          const mx_f32x16& c = acc[j / 2][pj];
          f32x4 y[2];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            float u = c[(j % 2) * 8 + i], w = c[(j % 2) * 8 + 4 + i];
            swap16(u, w);
            y[0][i] = u;
            y[1][i] = w;
          }
#pragma unroll
          for (int v = 0; v < 2; ++v) {
            const int row = 16 * v + r16, col = 16 * j + 4 * unit;
            if (wide) {
              float z[4] = {y[v].x, y[v].y, y[v].z, y[v].w};
              if (row < rows && col < left) mx_store4<OUT_BF16>(g.out, g.addend, (p0 + row) * g.ldo + q0 + col, left - col, z);
            } else {
              const f32x4 z = y[v] + a[j][v];
              if constexpr (OUT_BF16) store8(rsrc, u32x2{mx_pack_bf16x2(z.x, z.y), mx_pack_bf16x2(z.z, z.w)}, at(row, col, 2));
              else put(stream, __builtin_bit_cast(u32x4, z), at(row, col, 4));
            }
          }
        });
      };
      if (g.stream && counted) store_all(std::true_type{});
      else store_all(std::false_type{});
    });
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("" ::: "memory");
    if (!has_next) break;
    lid = next;
  }
}

// What is left of a T x T tile whose sums lie in LDS, rows T + 4 floats apart: the addend, the rounding, stores along rows.  A batch of rows'
// addends is requested before the first of them is stored.
template <int T, int THREADS, bool OUT_BF16>
FP4_D void finish_tile(const MxGemm& g, const float* tile, int64_t P0, int64_t Q0) {
  constexpr int UPR = T / 8, RPP = THREADS / UPR, NP = T / RPP, B = NP < 4 ? NP : 4;   // 8-column units a row, rows a pass, passes, passes a batch
  const int tid = threadIdx.x, ql = (tid % UPR) * 8;
  const int64_t q0 = Q0 + ql, left = g.Q - q0;
  if (left <= 0) return;
#pragma unroll 1
  for (int b = 0; b < NP; b += B) {
    float a[B][8];
#pragma unroll
    for (int i = 0; i < B; ++i) {
      const int64_t p = P0 + tid / UPR + (b + i) * RPP;
      if (g.addend && p < g.P) load_addend8(g, p * g.ldo + q0, left, a[i]);
      else
#pragma unroll
        for (int e = 0; e < 8; ++e) a[i][e] = 0.0f;
    }
#pragma unroll
    for (int i = 0; i < B; ++i) {
      const int pl = tid / UPR + (b + i) * RPP;
      const f32x4 u = *reinterpret_cast<const f32x4*>(&tile[pl * (T + 4) + ql]), v = *reinterpret_cast<const f32x4*>(&tile[pl * (T + 4) + ql + 4]);
      const float y[8] = {u.x + a[i][0], u.y + a[i][1], u.z + a[i][2], u.w + a[i][3], v.x + a[i][4], v.y + a[i][5], v.z + a[i][6], v.w + a[i][7]};
      if (P0 + pl < g.P) store8<OUT_BF16>(g, (P0 + pl) * g.ldo + q0, left, y);
    }
  }
}

// ---- 128 x 128 ------------------------------------------------------------------------------------------------------------------
// For outputs with too few 256 x 256 tiles.  Two groups of four waves, a wave 64 x 64 of the sums; the groups share each step, two of its
// four slices each, so that a SIMD has one wave that reads fragments while another multiplies (with four waves a step took
// the sum of both), and their sums are joined at the end, the first group's and the second's.  Steps go through a ring of four LDS stages
// with three on their way; scales come for two steps at a time, sixteen bytes of every row, into a ring of their own.  Bound by the loads'
// latency at the 96 KiB that a CU can have on their way: a step takes 0.68 - 0.72 us, 0.48 with the loads alone, 0.54 without them
// (2048 x 2048 over 2048 12.8 us, over 8192 in 8 x 4 bits 49; 498 x 11936 over 2024 in 8 x 4 bits 30.5).  Tried: the groups half a step apart,
// 55.3 against 53.2 us.
constexpr int MT = 128, M_RING = 4, M_WAVES = 8;
constexpr int M_OP = MT * BKB, M_STAGE = 2 * M_OP, M_LD = MT * 8 / (M_WAVES * 64), M_SC = M_RING * M_STAGE, M_SC_BYTES = 2 * MT * 16;
constexpr int M_SMEM = M_SC + M_RING * M_SC_BYTES;

template <bool OUT_BF16>
__global__ __launch_bounds__(M_WAVES * 64) void mx_gemm_mid_kernel(MxGemm g) {
  static_assert(M_RING * M_STAGE >= MT * (MT + 4) * 4 && M_SMEM <= 160 * 1024, "the sums lie over the ring");
  __shared__ __attribute__((aligned(16))) uint8_t smem[M_SMEM];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l32 = lane & 31, h = lane >> 5, group = wave >> 2;
  const int wp = (wave & 1) * 64, wq = (wave >> 1 & 1) * 64;
  // each XCD a contiguous run of tiles: of the whole output, or (first > 0) the quarters of the 256 x 256 tiles from `first` on
  const int per_xcd = (g.count + 7) / 8, id = (int)(blockIdx.x % 8) * per_xcd + (int)(blockIdx.x / 8);
  if ((int)(blockIdx.x / 8) >= per_xcd || id >= g.count) return;
  int tp, tq;
  if (g.first > 0) {
    tile_at(g, g.first + (id >> 2), tp, tq);
    tp = 2 * tp + (id & 1);
    tq = 2 * tq + (id >> 1 & 1);
  } else {
    tile_at(g, id, tp, tq);
  }
  const int64_t P0 = (int64_t)tp * MT, Q0 = (int64_t)tq * MT;
  if (P0 >= g.P || Q0 >= g.Q) return;   // a quarter behind the edge
  const int64_t rowb = g.pitch / 2, rows_s = g.pitch / MX_BLOCK, np = min(g.P - P0, (int64_t)MT), nq = min(g.Q - Q0, (int64_t)MT);
  const int KT = g.steps, T = KT * g.nl * g.nr;
  __amdgpu_buffer_rsrc_t rsrcL, rsrcR;
  auto planes = [&](int pass) {
    rsrcL = rows_rsrc(g.L + (pass % g.nl) * g.planeL + P0 * rowb, np, rowb);
    rsrcR = rows_rsrc(g.R + (pass / g.nl) * g.planeR + Q0 * rowb, nq, rowb);
  };
  planes(0);
  // waves 0, 1: L's scales, 2, 3: Rt's, 64 rows each; the second group has none to bring
  const bool scales_l = (wave & 2) == 0;
  const __amdgpu_buffer_rsrc_t rsrcS = scales_l ? rows_rsrc(g.sL + P0 * rows_s, np, rows_s) : rows_rsrc(g.sR + Q0 * rows_s, nq, rows_s);
  const uint32_t offS = (uint32_t)(min((int64_t)((wave & 1) * 64 + lane), (scales_l ? np : nq) - 1) * rows_s);
  uint32_t offL[M_LD], offR[M_LD];
#pragma unroll
  for (int j = 0; j < M_LD; ++j) {
    const int row = 8 * (wave * M_LD + j) + (lane >> 3), at = ((lane & 7) ^ ((row >> 1) & 7)) * 16;
    offL[j] = (uint32_t)(min((int64_t)row, np - 1) * rowb + at);   // rows past the edge re-read the last row
    offR[j] = (uint32_t)(min((int64_t)row, nq - 1) * rowb + at);
  }
  int ld_t = 0, ld_k = 0, ld_pass = 0, ld_pair = 0;
  auto request = [&]() {   // the next step; behind the last one zeros
    uint8_t* const st = smem + (ld_t & (M_RING - 1)) * M_STAGE;
    const bool in = ld_t < T;
    if ((ld_k & 1) == 0) {
      if (group == 0) to_lds16(rsrcS, smem + M_SC + (ld_pair & (M_RING - 1)) * M_SC_BYTES + wave * 1024, in ? offS : PAST_THE_END, ld_k * 8);
      ++ld_pair;
    }
#pragma unroll
    for (int j = 0; j < M_LD; ++j) {
      to_lds16(rsrcL, st + (wave * M_LD + j) * 1024, in ? offL[j] : PAST_THE_END, ld_k * BKB);
      to_lds16(rsrcR, st + M_OP + (wave * M_LD + j) * 1024, in ? offR[j] : PAST_THE_END, ld_k * BKB);
    }
    ++ld_t;
    if (++ld_k == KT) {
      ld_k = 0;
      if (++ld_pass < g.nl * g.nr) planes(ld_pass);
    }
  };
  const int key = (l32 >> 1) & 7;
  mx_f32x16 acc[2][2];
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int v = 0; v < 16; ++v) acc[i >> 1][i & 1][v] = 0.0f;
#pragma unroll
  for (int i = 0; i < M_RING - 1; ++i) request();
  uint32_t lessl = 0, lessr = 0;
  int rd_k = 0, rd_pass = 0, rd_pair = 0;
  const int slot0 = ((4 * h + 2 * group) ^ key) * 16, slot1 = ((4 * h + 2 * group + 1) ^ key) * 16;   // this group's two slices
  auto slices = [&](auto gc) {   // S: the first of the two
    constexpr int S = 2 * decltype(gc)::value;
    for (int t = 0; t < T; ++t) {
      asm volatile("" ::: "memory");
      // this wave's share of step t is there (at most the two steps behind it are not), and it is done reading step t - 1; behind the
      // barrier that holds for all
      constexpr int left = (M_RING - 2) * 2 * M_LD;
      __builtin_amdgcn_s_waitcnt(0x0070 | (left & 15) | ((left >> 4) << 14));
      __builtin_amdgcn_s_barrier();
      asm volatile("" ::: "memory");
      request();
      const uint8_t* const st = smem + (t & (M_RING - 1)) * M_STAGE;
      const uint8_t *const sL = st + (wp + l32) * BKB, *const sR = st + M_OP + (wq + l32) * BKB;
      const uint8_t* const sc = smem + M_SC + (rd_pair & (M_RING - 1)) * M_SC_BYTES + (rd_k & 1) * 8 + h * 4;
      uint32_t sl[2], sr[2];
      u32x4 fl[2][2], fr[2][2];
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        sl[j] = *reinterpret_cast<const uint32_t*>(sc + (wp + j * 32 + l32) * 16) - lessl;
        sr[j] = *reinterpret_cast<const uint32_t*>(sc + (MT + wq + j * 32 + l32) * 16) - lessr;
        fr[0][j] = *reinterpret_cast<const u32x4*>(sR + slot0 + j * 32 * BKB);
        fl[0][j] = *reinterpret_cast<const u32x4*>(sL + slot0 + j * 32 * BKB);
      }
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        fr[1][j] = *reinterpret_cast<const u32x4*>(sR + slot1 + j * 32 * BKB);
        fl[1][j] = *reinterpret_cast<const u32x4*>(sL + slot1 + j * 32 * BKB);
      }
      __builtin_amdgcn_sched_barrier(0);   // all requested before the first product
#pragma unroll
      for (int qi = 0; qi < 2; ++qi)
#pragma unroll
        for (int pj = 0; pj < 2; ++pj) acc[qi][pj] = mx_mfma<S>(fr[0][qi], fl[0][pj], acc[qi][pj], sr[qi], sl[pj]);
#pragma unroll
      for (int qi = 0; qi < 2; ++qi)
#pragma unroll
        for (int pj = 0; pj < 2; ++pj) acc[qi][pj] = mx_mfma<S + 1>(fr[1][qi], fl[1][pj], acc[qi][pj], sr[qi], sl[pj]);
      rd_pair += rd_k & 1;
      if (++rd_k == KT) {
        rd_pair += rd_k & 1;
        rd_k = 0;
        ++rd_pass;
        lessl = rd_pass % g.nl ? MX_EIGHTH : 0u;
        lessr = rd_pass / g.nl ? MX_EIGHTH : 0u;
      }
    }
  };
  if (group == 0) slices(std::integral_constant<int, 0>{});
  else slices(std::integral_constant<int, 1>{});
  __builtin_amdgcn_s_waitcnt(0);   // no load may land over the sums
  __syncthreads();
  float* const tile = reinterpret_cast<float*>(smem);
  auto each = [&](auto&& f) {
#pragma unroll
    for (int pj = 0; pj < 2; ++pj)
#pragma unroll
      for (int qi = 0; qi < 2; ++qi)
#pragma unroll
        for (int b = 0; b < 4; ++b) {
          const mx_f32x16& c = acc[qi][pj];
          f(f32x4{c[b * 4], c[b * 4 + 1], c[b * 4 + 2], c[b * 4 + 3]},
            *reinterpret_cast<f32x4*>(&tile[(wp + pj * 32 + l32) * (MT + 4) + wq + qi * 32 + b * 8 + h * 4]));
        }
  };
  if (group == 1) each([](const f32x4& v, f32x4& at) { at = v; });
  __syncthreads();
  if (group == 0) each([](const f32x4& v, f32x4& at) { at = v + at; });
  __syncthreads();
  finish_tile<MT, M_WAVES * 64, OUT_BF16>(g, tile, P0, Q0);
}

// ---- 32 x 32, the contraction shared ---------------------------------------------------------------------------------------------
// For the smallest outputs: a workgroup of four waves takes 32 x 32, and each wave every fourth step of the contraction through a ring of its
// own, without a barrier before the end.  Such a call is one round trip to memory after another, so there are as many workgroups as can be
// and each wave has RING steps under way.  The waves' sums are added in their order.  512 x 512 over 256 in 8 x 4 bits 5.1 us, a launch by itself
// 3.4; 1024 x 1024 over 4096 15.5, where what bounds it are the operands' reads from L2 (32 rows and 32 columns a tile).
constexpr int ST = 32, S_OP = ST * BKB, S_STEP = 2 * S_OP + 512, S_LD = ST / 8;

template <bool OUT_BF16, int RING>
__global__ __launch_bounds__(256) void mx_gemm_split_kernel(MxGemm g) {
  constexpr int LD = ST + 4, WAVES = 4;
  __shared__ __attribute__((aligned(16))) uint8_t smem[WAVES * RING * S_STEP];
  static_assert(RING * S_STEP >= ST * LD * 4, "a wave's sums lie over its ring");
  auto part = [&](int w) { return reinterpret_cast<float*>(smem + w * (RING * S_STEP)); };
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l32 = lane & 31, h = lane >> 5;
  // each XCD a contiguous run of tiles, column by column: the rows of Rt are read by one of them
  const int per_xcd = (g.count + 7) / 8, id = (int)(blockIdx.x % 8) * per_xcd + (int)(blockIdx.x / 8);
  if ((int)(blockIdx.x / 8) >= per_xcd || id >= g.count) return;
  const int64_t P0 = (int64_t)(id % g.tiles_p) * ST, Q0 = (int64_t)(id / g.tiles_p) * ST;
  const int64_t rowb = g.pitch / 2, rows_s = g.pitch / MX_BLOCK, np = min(g.P - P0, (int64_t)ST), nq = min(g.Q - Q0, (int64_t)ST);
  const int KT = g.steps, T = KT * g.nl * g.nr, steps = (T - wave + WAVES - 1) / WAVES;   // of this wave
  const __amdgpu_buffer_rsrc_t rsrcSL = rows_rsrc(g.sL + P0 * rows_s, np, rows_s), rsrcSR = rows_rsrc(g.sR + Q0 * rows_s, nq, rows_s);
  uint32_t offL[S_LD], offR[S_LD];
#pragma unroll
  for (int j = 0; j < S_LD; ++j) {
    const int row = 8 * j + (lane >> 3), at = ((lane & 7) ^ ((row >> 1) & 7)) * 16;
    offL[j] = (uint32_t)(min((int64_t)row, np - 1) * rowb + at);   // rows past the edge re-read the last row
    offR[j] = (uint32_t)(min((int64_t)row, nq - 1) * rowb + at);
  }
  const uint32_t offSL = (uint32_t)(min((int64_t)l32, np - 1) * rows_s + h * 4), offSR = (uint32_t)(min((int64_t)l32, nq - 1) * rows_s + h * 4);
  uint8_t* const mine = smem + wave * (RING * S_STEP);
  auto request = [&](int i) {   // steps past the last arrive as zeros
    uint8_t* const st = mine + (i % RING) * S_STEP;
    const bool in = i < steps;
    const int t = in ? wave + WAVES * i : 0, pass = t / KT, k = t - pass * KT;
    const __amdgpu_buffer_rsrc_t rsrcL = rows_rsrc(g.L + (pass % g.nl) * g.planeL + P0 * rowb, np, rowb);
    const __amdgpu_buffer_rsrc_t rsrcR = rows_rsrc(g.R + (pass / g.nl) * g.planeR + Q0 * rowb, nq, rowb);
#pragma unroll
    for (int j = 0; j < S_LD; ++j) {
      to_lds16(rsrcL, st + j * 1024, in ? offL[j] : PAST_THE_END, k * BKB);
      to_lds16(rsrcR, st + S_OP + j * 1024, in ? offR[j] : PAST_THE_END, k * BKB);
    }
    to_lds4(rsrcSL, st + 2 * S_OP, in ? offSL : PAST_THE_END, k * 8);
    to_lds4(rsrcSR, st + 2 * S_OP + 256, in ? offSR : PAST_THE_END, k * 8);
  };
  const int key = (l32 >> 1) & 7;
  mx_f32x16 acc;
#pragma unroll
  for (int v = 0; v < 16; ++v) acc[v] = 0.0f;
#pragma unroll
  for (int i = 0; i < RING; ++i) request(i);
  for (int i = 0; i < steps; ++i) {
    asm volatile("" ::: "memory");
    constexpr int left = (RING - 1) * (2 * S_LD + 2);   // the steps behind this one
    __builtin_amdgcn_s_waitcnt(0x0070 | (left & 15) | ((left >> 4) << 14));
    asm volatile("" ::: "memory");
    const uint8_t* const st = mine + (i % RING) * S_STEP;
    const int pass = (wave + WAVES * i) / KT;
    const uint32_t sl = *reinterpret_cast<const uint32_t*>(st + 2 * S_OP + lane * 4) - (pass % g.nl ? MX_EIGHTH : 0u);
    const uint32_t sr = *reinterpret_cast<const uint32_t*>(st + 2 * S_OP + 256 + lane * 4) - (pass / g.nl ? MX_EIGHTH : 0u);
    u32x4 fl[4], fr[4];
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      const int slot = l32 * BKB + ((4 * h + s) ^ key) * 16;
      fr[s] = *reinterpret_cast<const u32x4*>(st + S_OP + slot);
      fl[s] = *reinterpret_cast<const u32x4*>(st + slot);
    }
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // read: the slot may be filled again
    request(i + RING);
    __builtin_amdgcn_sched_barrier(0);
    static_for<4>([&](auto sc) {
      constexpr int s = decltype(sc)::value;
      acc = mx_mfma<s>(fr[s], fl[s], acc, sr, sl);
    });
  }
  __builtin_amdgcn_s_waitcnt(0);   // no load may land over the sums
#pragma unroll
  for (int b = 0; b < 4; ++b)
    *reinterpret_cast<f32x4*>(&part(wave)[l32 * LD + b * 8 + h * 4]) = f32x4{acc[b * 4], acc[b * 4 + 1], acc[b * 4 + 2], acc[b * 4 + 3]};
  __syncthreads();
  const int row = tid >> 3, col = (tid & 7) * 4;   // four columns of a row a thread
  f32x4 sum = *reinterpret_cast<const f32x4*>(&part(0)[row * LD + col]);
#pragma unroll
  for (int w = 1; w < WAVES; ++w) sum += *reinterpret_cast<const f32x4*>(&part(w)[row * LD + col]);
  float y[4] = {sum.x, sum.y, sum.z, sum.w};
  if (P0 + row < g.P && Q0 + col < g.Q) mx_store4<OUT_BF16>(g.out, g.addend, (P0 + row) * g.ldo + Q0 + col, g.Q - Q0 - col, y);
}

void set_tiles(MxGemm& g, int rows, int cols) {
  g.tiles_p = (int)((g.P + rows - 1) / rows);
  g.tiles_q = (int)((g.Q + cols - 1) / cols);
  g.first = 0;
  g.count = g.tiles_p * g.tiles_q;
}

template <bool OUT_BF16>
int launch(MxGemm& g, MxTiling t, int n_cu, hipStream_t s) {
  const auto resident = [&](int count) { return dim3((unsigned)std::min((count + 7) / 8 * 8, n_cu / 8 * 8)); };   // a workgroup a CU
  const auto dealt = [](int count) { return dim3((unsigned)((count + 7) / 8 * 8)); };   // a run of tiles for each XCD
  if (t.tile == 256) {
    set_tiles(g, 256, 256);
    MxGemm m = g;
    g.count -= t.rest;
    hipLaunchKernelGGL((mx_gemm_big_kernel<256, OUT_BF16>), resident(g.count), dim3(BWAVES * 64), 0, s, g);
    if (t.rest) {
      m.first = g.count;
      m.count = 4 * t.rest;
      hipLaunchKernelGGL((mx_gemm_mid_kernel<OUT_BF16>), dealt(m.count), dim3(M_WAVES * 64), 0, s, m);
    }
  } else if (t.tile == 192) {
    set_tiles(g, 256, 192);
    hipLaunchKernelGGL((mx_gemm_big_kernel<192, OUT_BF16>), resident(g.count), dim3(BWAVES * 64), 0, s, g);
  } else if (t.tile == 128) {
    set_tiles(g, 128, 128);
    hipLaunchKernelGGL((mx_gemm_mid_kernel<OUT_BF16>), dealt(g.count), dim3(M_WAVES * 64), 0, s, g);
  } else if (t.tile == 32) {
    set_tiles(g, 32, 32);
    if (g.count <= n_cu) hipLaunchKernelGGL((mx_gemm_split_kernel<OUT_BF16, 4>), dealt(g.count), dim3(256), 0, s, g);
    else hipLaunchKernelGGL((mx_gemm_split_kernel<OUT_BF16, 2>), dealt(g.count), dim3(256), 0, s, g);
  } else {
    const dim3 grid((unsigned)((g.P + 63) / 64), (unsigned)((g.Q + 63) / 64));
    hipLaunchKernelGGL((mx_gemm_small_kernel<OUT_BF16>), grid, dim3(256), 0, s, g);
  }
  FP4_CHECK_LAUNCH();
  return FP4_OK;
}

}  // namespace

// P and Q are at least 1; Kc may be 0.  tile: one of MxTiling's, or 0 for the rule's.
int mx_launch_gemm(const uint8_t* L, const uint8_t* sL, int bits_l, const uint8_t* R, const uint8_t* sR, int bits_r, int64_t P, int64_t Q, int64_t Kc,
                   const float* addend, void* out, int out_bf16, int64_t ldo, int tile, hipStream_t s) {
  const int n_cu = fp4_compute_units_of_current_device();
  MxTiling t = mx_gemm_tiling(P, Q, Kc, bits_l, bits_r, n_cu);
  if (tile) t = {tile, 0};
  if (t.tile == 16) return mx_launch_few(L, sL, nullptr, 0, 0, bits_l, R, sR, bits_r, P, Q, Kc, addend, out, out_bf16, ldo, s);
  MxGemm g;
  g.L = L; g.R = R; g.sL = sL; g.sR = sR;
  g.addend = addend;
  g.out = out;
  g.P = P; g.Q = Q; g.ldo = ldo;
  g.pitch = mx_pitch_of(Kc);
  g.steps = (int)((Kc + 255) / 256);
  g.planeL = P * (g.pitch / 2);
  g.planeR = Q * (g.pitch / 2);
  // An output beyond the 256 MiB of the last-level cache only takes the operands' place there: 16384 x 12288 in bf16 430 us past the caches,
  // 480 through them; 8192 x 11008 212 and 209, 4096 x 4096 in fp32 134 and 127.
  g.stream = P * Q * (out_bf16 ? 2 : 4) > (int64_t)256 << 20;
  g.nl = bits_l / 4;
  g.nr = bits_r / 4;
  return out_bf16 ? launch<true>(g, t, n_cu, s) : launch<false>(g, t, n_cu, s);
}

// For measuring and for tests: the product by one kind of tile (16, 32, 64, 128, 192 or 256), or by the rule's (0).
extern "C" int mx_gemm_by_tile(const fp4_mx* l, const fp4_mx* rt, const float* addend, void* out, fp4_dtype out_dt, int64_t ldo, int tile, void* stream) {
  if (tile != 0 && tile != 16 && tile != 32 && tile != 64 && tile != 128 && tile != 192 && tile != 256) return FP4_ERR_ARG;
  const int rc = mx_check_gemm(l, rt, addend, out, out_dt, ldo);
  if (rc || l->lines == 0 || rt->lines == 0) return rc;
  return mx_launch_gemm(l->codes, l->scales, l->bits, rt->codes, rt->scales, rt->bits, l->lines, rt->lines, l->length, addend, out, out_dt == FP4_BF16, ldo,
                        l->length == 0 ? 0 : tile, (hipStream_t)stream);
}

extern "C" int mx_gemm_tile(int64_t P, int64_t Q, int64_t Kc, int bits_l, int bits_r, int compute_units, int* last_round) {
  if (P <= 0 || Q <= 0 || Kc < 0 || compute_units < 8) return FP4_ERR_SHAPE;
  const MxTiling t = mx_gemm_tiling(P, Q, Kc, bits_l, bits_r, compute_units);
  if (last_round) *last_round = t.rest;
  return t.tile;
}
