// Tiles of 16-bit matrix products on the gfx950 matrix cores, both operands along the contraction:
//
//   acc[p, q] = sum over k of L[p, k] R[q, k]
//
// fp32 sums of exact products.  What becomes of a tile is its epilogue's (hp_head.hip).
//
// v_mfma_f32_16x16x32: lane (l16, g) brings elements 8 g .. 8 g + 7 of row l16 of either operand.  A step is 64 elements, 128 bytes, of a row, in two
// slices.  Result: lane (l16, g) holds, of row l16 of L, columns 4 g + e of the block, in register e.  (The 32 x 32 x 16 instruction reads half of the
// operands for the same products, and yet draws more power, which is what bounds large products: 16384 x 4096 over 8192 895 against 829 us.)
//
// Operands come into LDS by direct loads, a ring of NST steps.  A row takes 128 bytes of a stage, its 16-byte chunk c in slot c ^ ((row >> 1) & 7),
// so that sixteen rows reading one chunk touch sixteen different bank groups.  Chunks behind K arrive as zeros, rows behind the matrix's edge repeat its last one.
#pragma once
#include "hp_common.h"

#include <type_traits>
#include <utility>

typedef __bf16 hp_bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 hp_f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 hp_f16x2 __attribute__((ext_vector_type(2)));
typedef float hp_f32x16 __attribute__((ext_vector_type(16)));

struct HpOperands {
  const uint16_t *L, *R;
  int64_t P, Q, K;          // K a multiple of 8
  int64_t ldL, ldR;         // at most 2^21
  int tiles_p, tiles_q;
  int splits, split_steps;  // the contraction is cut into so many parts of so many steps
};

template <int N, class F, int... I>
FP4_D void hp_static_for_impl(F&& f, std::integer_sequence<int, I...>) { (f(std::integral_constant<int, I>{}), ...); }
template <int N, class F>
FP4_D void hp_static_for(F&& f) { hp_static_for_impl<N>(f, std::make_integer_sequence<int, N>{}); }

// WP x WQ waves of PJ x QI blocks of 16 x 16, a ring of NST stages.
template <int WP_, int WQ_, int PJ_, int QI_, int NST_>
struct HpShape {
  static constexpr int WP = WP_, WQ = WQ_, PJ = PJ_, QI = QI_, NST = NST_;
  static constexpr int WAVES = WP * WQ, BP = WP * PJ * 16, BQ = WQ * QI * 16;
  static constexpr int LDL = BP / 8 / WAVES, LDR = BQ / 8 / WAVES, LOADS = LDL + LDR;   // of 64 chunks of 16 bytes, a wave and step
  static constexpr int OP_L = BP * 128, STAGE = (BP + BQ) * 128, SMEM = NST * STAGE;
  static_assert(LDL * 8 * WAVES == BP && LDR * 8 * WAVES == BQ, "rows a load");
  static_assert(SMEM <= 160 * 1024, "LDS");
};

constexpr uint32_t HP_PAST_THE_END = 0xf0000000u;   // behind any descriptor: arrives as zeros
constexpr int HP_GROUP_P = 4;                       // tile rows side by side

FP4_D const uint8_t* hp_uniform(const void* p) {
  const uint64_t v = (uint64_t)p;
  const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)v), hi = __builtin_amdgcn_readfirstlane((uint32_t)(v >> 32));
  return (const uint8_t*)(((uint64_t)hi << 32) | lo);
}
FP4_D __amdgpu_buffer_rsrc_t hp_rsrc(const void* p, int64_t bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(hp_uniform(p)), 0, __builtin_amdgcn_readfirstlane((int)bytes), 0x00020000);
}
FP4_D void hp_to_lds(__amdgpu_buffer_rsrc_t rsrc, uint8_t* lds, uint32_t voff, int soff) {   // a wave's lanes one behind another from `lds` on
  __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (__attribute__((address_space(3))) void*)lds, 16, voff, soff, 0, 0);
}
// Until all but the latest N requests of this wave have landed, and its reads of LDS are over.
template <int N>
FP4_D void hp_wait() {
  static_assert(N < 64, "what the counter holds");
  __builtin_amdgcn_s_waitcnt(0x0070 | (N & 15) | ((N >> 4) << 14));
}
template <bool F16>
FP4_D f32x4 hp_mfma(const u32x4& r, const u32x4& l, const f32x4& c) {
  if constexpr (F16) return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(hp_f16x8, r), __builtin_bit_cast(hp_f16x8, l), c, 0, 0, 0);
  else return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(hp_bf16x8, r), __builtin_bit_cast(hp_bf16x8, l), c, 0, 0, 0);
}
FP4_D hp_f32x16 hp_mfma32(const u32x4& r, const u32x4& l, const hp_f32x16& c) {   // bf16, 32 x 32 x 16
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(hp_bf16x8, r), __builtin_bit_cast(hp_bf16x8, l), c, 0, 0, 0);
}
// Between the lanes' four groups of sixteen: the second and fourth group of a with the first and third of b; the upper two groups of a with
// the lower two of b.
FP4_D void hp_swap16(uint32_t& a, uint32_t& b) {
  const auto r = __builtin_amdgcn_permlane16_swap(a, b, false, false);
  a = r[0]; b = r[1];
}
FP4_D void hp_swap32(uint32_t& a, uint32_t& b) {
  const auto r = __builtin_amdgcn_permlane32_swap(a, b, false, false);
  a = r[0]; b = r[1];
}
FP4_D float hp_other_half(float v) {   // of the lane 32 further
  uint32_t a = f2u(v), b = a;
  hp_swap32(a, b);
  return u2f((threadIdx.x & 32) ? a : b);
}
FP4_D float hp_other_sixteen(float v) {   // of the lane 16 further in its half
  uint32_t a = f2u(v), b = a;
  hp_swap16(a, b);
  return u2f((threadIdx.x & 16) ? a : b);
}

// A workgroup's tile and its part of the contraction.  Workgroups go round the eight XCDs; each XCD takes a contiguous run of tiles, so
// that those that share rows meet in one L2.
struct HpTile { int tp, tq, split; };
FP4_D HpTile hp_tile_at(const HpOperands& g) {
  const int n = g.tiles_p * g.tiles_q * g.splits, per = n / 8, more = n % 8;
  const int xcd = blockIdx.x % 8, i = blockIdx.x / 8;
  const int id = xcd * per + min(xcd, more) + i;
  HpTile t;
  const int tiles = g.tiles_p * g.tiles_q, tile = id % tiles;
  t.split = id / tiles;
  const int in_group = HP_GROUP_P * g.tiles_q, first = tile / in_group * HP_GROUP_P, size = min(g.tiles_p - first, HP_GROUP_P);
  t.tp = first + tile % in_group % size;
  t.tq = tile % in_group / size;
  return t;
}

// The sums of one tile.  smem is free of requests and of other waves' reads when it returns.  watch sees each slice's fragments.
// A slice's fragments are read while the matrix cores work on the slice before.  A step's barrier stands between its slices: by then every wave holds the
// second slice's fragments, so that the stage is free for a later step, and the next step has landed, whose first fragments are read in the second slice's shadow.
// The steady loop has no branches, and requests and reads stand one by one among the products: with the compiler's own order, all reads ahead of all
// products, 8192 x 8192 over 4096 takes 449 us in 256 x 256 tiles and 2048 x 2048 over 4096 takes 52 in 128 x 128 ones; so 418 and 42.  Requests behind
// the reads gain another us there, but lose 5 % where rows lie 128 KiB apart and what is asked for comes late.
template <class S, bool F16, class Watch>
FP4_D void hp_tile_sums(const HpOperands& g, const HpTile& tile, uint8_t* smem, f32x4 (&acc)[S::QI][S::PJ], Watch&& watch) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int l16 = lane & 15, quarter = lane >> 4;
  const int64_t P0 = (int64_t)tile.tp * S::BP, Q0 = (int64_t)tile.tq * S::BQ;
  const int64_t rowL = g.ldL * 2, rowR = g.ldR * 2;
  const __amdgpu_buffer_rsrc_t rsrcL = hp_rsrc(g.L + P0 * g.ldL, min(g.P - P0, (int64_t)S::BP) * rowL);
  const __amdgpu_buffer_rsrc_t rsrcR = hp_rsrc(g.R + Q0 * g.ldR, min(g.Q - Q0, (int64_t)S::BQ) * rowR);
  uint32_t offL[S::LDL], offR[S::LDR];
  const auto chunk_of = [&](int row) { return (lane & 7) ^ ((row >> 1) & 7); };
#pragma unroll
  for (int j = 0; j < S::LDL; ++j) {
    const int row = 8 * (wave * S::LDL + j) + (lane >> 3);
    offL[j] = (uint32_t)((min(P0 + row, g.P - 1) - P0) * rowL + chunk_of(row) * 16);
  }
#pragma unroll
  for (int j = 0; j < S::LDR; ++j) {
    const int row = 8 * (wave * S::LDR + j) + (lane >> 3);
    offR[j] = (uint32_t)((min(Q0 + row, g.Q - 1) - Q0) * rowR + chunk_of(row) * 16);
  }
  const int first = tile.split * g.split_steps, all = (int)((g.K + 63) / 64), T = min(all - first, g.split_steps);
  const auto load_step = [&](int t, auto whole) {
    const int step = first + t;
    uint8_t* const stage = smem + t % S::NST * S::STAGE;
    const int left = (int)(g.K / 8) - step * 8;   // chunks of a row from here on
    if (decltype(whole)::value || left >= 8) {
#pragma unroll
      for (int j = 0; j < S::LDL; ++j) hp_to_lds(rsrcL, stage + (wave * S::LDL + j) * 1024, offL[j], step * 128);
#pragma unroll
      for (int j = 0; j < S::LDR; ++j) hp_to_lds(rsrcR, stage + S::OP_L + (wave * S::LDR + j) * 1024, offR[j], step * 128);
    } else {
#pragma unroll
      for (int j = 0; j < S::LDL; ++j)
        hp_to_lds(rsrcL, stage + (wave * S::LDL + j) * 1024, chunk_of(8 * (wave * S::LDL + j) + (lane >> 3)) < left ? offL[j] : HP_PAST_THE_END, step * 128);
#pragma unroll
      for (int j = 0; j < S::LDR; ++j)
        hp_to_lds(rsrcR, stage + S::OP_L + (wave * S::LDR + j) * 1024, chunk_of(8 * (wave * S::LDR + j) + (lane >> 3)) < left ? offR[j] : HP_PAST_THE_END,
                  step * 128);
    }
  };
  const int key = (l16 >> 1) & 7, wave_p = wave % S::WP, wave_q = wave / S::WP;
  const int at_l = (wave_p * (S::PJ * 16) + l16) * 128, at_r = S::OP_L + (wave_q * (S::QI * 16) + l16) * 128;
#pragma unroll
  for (int i = 0; i < S::QI; ++i)
#pragma unroll
    for (int j = 0; j < S::PJ; ++j) acc[i][j] = f32x4{0, 0, 0, 0};
  if (T <= 0) return;
  u32x4 fl[2][S::PJ], fr[2][S::QI];
  const auto read = [&](int t, int s) {
    const uint8_t* const stage = smem + t % S::NST * S::STAGE + ((4 * s + quarter) ^ key) * 16;
#pragma unroll
    for (int j = 0; j < S::QI; ++j) fr[s][j] = *reinterpret_cast<const u32x4*>(stage + at_r + j * 16 * 128);
#pragma unroll
    for (int j = 0; j < S::PJ; ++j) fl[s][j] = *reinterpret_cast<const u32x4*>(stage + at_l + j * 16 * 128);
  };
  const auto multiply = [&](int s) {
#pragma unroll
    for (int i = 0; i < S::QI; ++i)
#pragma unroll
      for (int j = 0; j < S::PJ; ++j) acc[i][j] = hp_mfma<F16>(fr[s][i], fl[s][j], acc[i][j]);
    watch(fl[s], fr[s]);
  };
#pragma unroll
  for (int t = 0; t < S::NST; ++t)
    if (t < T) load_step(t, std::false_type{});
  if (T >= S::NST) hp_wait<(S::NST - 1) * S::LOADS>();
  else hp_wait<0>();
  __builtin_amdgcn_s_barrier();   // a bare one: a fence would wait for the other stages too
  asm volatile("" ::: "memory");
  read(0, 0);
  constexpr int BETWEEN = S::PJ * S::QI >= 32 ? 2 : 1;
  const auto reads_among = [] {   // a read, a product, a read, ...
    hp_static_for<S::PJ + S::QI>([](auto) {
      __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
      __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
    });
  };
  const auto requests_among = [] {
    hp_static_for<S::LOADS>([](auto) {
      __builtin_amdgcn_sched_group_barrier(0x020, 1, 0);
      __builtin_amdgcn_sched_group_barrier(0x008, BETWEEN, 0);
    });
  };
  const auto step = [&](int t, auto steady) {
    constexpr bool STEADY = decltype(steady)::value;
    read(t, 1);
    multiply(0);
    if constexpr (STEADY) {
      reads_among();
      __builtin_amdgcn_sched_barrier(0);
    }
    asm volatile("" ::: "memory");
    // Steps t + 2 .. t + NST - 1 may still be on their way; towards the end there are fewer, and then all have to have landed
    if (STEADY || t + S::NST - 1 < T) hp_wait<(S::NST - 2) * S::LOADS>();
    else hp_wait<0>();
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    if (STEADY || t + S::NST < T) load_step(t + S::NST, steady);
    if (STEADY || t + 1 < T) read(t + 1, 0);
    multiply(1);
    if constexpr (STEADY) {
      requests_among();
      reads_among();
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  int t = 0;
  for (; t < T - S::NST - 1; ++t) step(t, std::true_type{});   // free of branches: the steps it requests are whole ones
  for (; t < T; ++t) step(t, std::false_type{});
  __syncthreads();
}
