// The head: logits, softmax cross entropy and its gradients, the vocabulary in pieces.
//
//   z = x w^T,  lse_t = log sum_v e^z[t, v],  loss_t = lse_t - z[t, target_t]
//   dz[t, v] = c_t (e^(z[t, v] - lse_t) - [v = target_t]),  c_t the gradient of loss_t;   dx = dz w,  dw = dz^T x
//
// Forward: tiles of z in registers, of which a tile leaves each row's maximum m and sum of e^(z - m), and the target's z; a second launch joins the tiles
// in their order.  A sum of 0 is that of no columns, or of logits of -inf; one that is NaN (a logit of NaN or +inf) is carried on into the row's lse and loss.
// Backward, a piece of the vocabulary at a time: its logits again, of which e^(z - lse) - [target] is kept as fp16 under 2^15 (11 bits; its
// values lie in [-1, 1], and below 2^-29 of 1 an element loses bits, below 2^-40 all of them); dx adds the product with the piece of w, dw's rows are the product
// with c x.  Both contract over what lies across in memory, so transposed copies are made, and as they are made anyway they are made in fp16, under
// a power of two that brings their largest element to [2^14, 2^15): w's bf16 keep all their bits unless they lie 2^-31 below it, c x is rounded
// to 11 bits.  (With bf16 operands the products' error would be that of the bf16 outputs' own rounding over again.)  Sums are fp32.
#include "hp_gemm.h"

#include <algorithm>
#include <cstdint>

namespace {

constexpr float LOG2E = 1.44269504088896340736f, LN2 = 0.693147180559945309417f;
constexpr float DZ_SCALE = 32768.0f;   // of e^(z - lse) - [target] in fp16

// The power of two that brings a largest magnitude (its bits) to [2^14, 2^15), and its inverse.  Held in what fp32 has both of.
FP4_D float scale_of(uint32_t amax, bool inverse) {
  int e = 14 + 127 - (int)(amax >> 23);
  e = amax == 0 ? 0 : max(-126, min(126, e));
  return u2f((uint32_t)(127 + (inverse ? -e : e)) << 23);
}

enum { EPI_STATS, EPI_DZ, EPI_ADD, EPI_OUT };

struct HeadTile {
  HpOperands g;
  const int64_t* targets;
  int64_t first, V;          // the piece's first row of w, all rows
  float2* part;              // STATS: [tiles_q][P] maximum and sum
  float* target_z;           // STATS: [P]
  const float* lse;          // DZ
  uint16_t *dz, *dz_across;  // DZ: [P x ld], zeros from Q to ld; [Q x ld_across], zeros from P to the next multiple of 8 at least.  Either may be NULL
  int64_t ld, ld_across;
  float* sums;               // ADD: [splits][P x Q]
  bool add;                  // ADD, OUT: to what is there
  const uint32_t* amax;      // ADD, OUT: of the operand under a power of two
  void* out;                 // OUT
  bool out_bf16;
  uint32_t *amax_w, *amax_x; // DZ: largest magnitudes of w's piece and of c x, bits, 0 before; either may be NULL
  const float* dloss;        // c
};

template <class S>
FP4_D void stats_epilogue(const HeadTile& a, const HpTile& tile, uint8_t* smem, const f32x4 (&acc)[S::QI][S::PJ]) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l16 = lane & 15, quarter = lane >> 4;
  const int wave_p = wave % S::WP, wave_q = wave / S::WP;
  const int64_t q0 = (int64_t)tile.tq * S::BQ + wave_q * (S::QI * 16), left = a.g.Q - q0;
  float2* const lds = reinterpret_cast<float2*>(smem);   // [WQ][BP]
#pragma unroll
  for (int pj = 0; pj < S::PJ; ++pj) {
    const int row = wave_p * (S::PJ * 16) + pj * 16 + l16;
    const int64_t p = (int64_t)tile.tp * S::BP + row;
    const int64_t t = p < a.g.P ? a.targets[p] : -1;
    float m = -INFINITY;
    if (left >= S::QI * 16) {
#pragma unroll
      for (int i = 0; i < S::QI; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) m = fmaxf(m, acc[i][pj][e]);
    } else {
#pragma unroll
      for (int i = 0; i < S::QI; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) m = i * 16 + quarter * 4 + e < left ? fmaxf(m, acc[i][pj][e]) : m;
    }
    m = fmaxf(m, hp_other_sixteen(m));
    m = fmaxf(m, hp_other_half(m));
    const float ml = m == -INFINITY ? 0.0f : m * LOG2E;   // of nothing, or nothing finite
    float s = 0.0f;
#pragma unroll
    for (int i = 0; i < S::QI; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float x = __builtin_amdgcn_exp2f(fmaf(acc[i][pj][e], LOG2E, -ml));
        s += i * 16 + quarter * 4 + e < left ? x : 0.0f;
      }
    s += hp_other_sixteen(s);
    s += hp_other_half(s);
    if (quarter == 0) lds[wave_q * S::BP + row] = float2{m, s};
    const bool here = t >= q0 && t < q0 + std::min<int64_t>(left, S::QI * 16);
    if (__ballot(here)) {
      const int at = (int)(t - q0);
#pragma unroll
      for (int i = 0; i < S::QI; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (here && at == i * 16 + quarter * 4 + e) a.target_z[p] = acc[i][pj][e];
    }
  }
  __syncthreads();
  for (int row = threadIdx.x; row < S::BP; row += S::WAVES * 64) {
    const int64_t p = (int64_t)tile.tp * S::BP + row;
    if (p >= a.g.P) break;
    float m = lds[row].x;
#pragma unroll
    for (int i = 1; i < S::WQ; ++i) m = fmaxf(m, lds[i * S::BP + row].x);
    float s = 0.0f;
#pragma unroll
    for (int i = 0; i < S::WQ; ++i) {
      const float2 o = lds[i * S::BP + row];
      // A wave's terms carry 2^off in common: what the rounding of its m log2 e left
      const float off = fmaf(o.x, LOG2E, -(o.x * LOG2E));
      if (o.y != 0.0f) s += o.y * __builtin_amdgcn_exp2f((o.x - m) * LOG2E - off);   // NaN too
    }
    if (s > 0.0f && s < 1.0f) s = 1.0f;   // it holds the maximum's own term, so that no loss falls below 0
    a.part[(int64_t)tile.tq * a.g.P + p] = float2{m, s};
  }
}

FP4_D uint32_t pack_f16(float a, float b) {
  const hp_f16x2 v = {(_Float16)a, (_Float16)b};
  return __builtin_bit_cast(uint32_t, v);
}

// A row's four columns of one 16 x 16 block (a) and of the block beside it (b), two words each -> eight columns in a row: 8 unit on of the two blocks' 32,
// unit = lane / 32 + 2 (lane / 16 % 2), so that a store is 64 bytes of a row.
FP4_D u32x4 eight_columns(uint32_t a0, uint32_t a1, uint32_t b0, uint32_t b1) {
  hp_swap16(a0, b0);
  hp_swap16(a1, b1);
  return u32x4{a0, a1, b0, b1};
}
FP4_D uint32_t from_lane(uint32_t x, std::integral_constant<int, 1>) { return (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0xB1, 0xf, 0xf, true); }   // lane ^ 1
FP4_D uint32_t from_lane(uint32_t x, std::integral_constant<int, 2>) { return (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0x4E, 0xf, 0xf, true); }   // lane ^ 2
// Four lanes' rows of four 16-bit columns (two words) -> lane k of them has column k of the four rows.
FP4_D u32x2 turn_four(uint32_t a, uint32_t b) {
  const int lane = threadIdx.x & 3;
  const uint32_t choose = lane & 1 ? 0x03020706u : 0x05040100u;   // bytes of {the neighbour's word, its own}
  const uint32_t x = __builtin_amdgcn_perm(from_lane(a, std::integral_constant<int, 1>{}), a, choose);   // column 0 or 1 of two rows
  const uint32_t y = __builtin_amdgcn_perm(from_lane(b, std::integral_constant<int, 1>{}), b, choose);   // column 2 or 3
  const uint32_t got = from_lane(lane & 2 ? x : y, std::integral_constant<int, 2>{});
  return lane & 2 ? u32x2{got, y} : u32x2{x, got};
}
FP4_D uint32_t from_lane(uint32_t x, std::integral_constant<int, 4>) {   // lane ^ 4: ^ 7 and then ^ 3
  return (uint32_t)__builtin_amdgcn_mov_dpp(__builtin_amdgcn_mov_dpp((int)x, 0x141, 0xf, 0xf, true), 0x1B, 0xf, 0xf, true);
}
// Four rows of a column in each of two blocks of sixteen rows -> eight rows in a row of one of them, the first block's in lanes without bit 2.
FP4_D u32x4 eight_rows(u32x2 a, u32x2 b) {
  const bool second = threadIdx.x & 4;
  const std::integral_constant<int, 4> four;
  const u32x2 own = second ? b : a, others = second ? a : b;
  const u32x2 got = {from_lane(others.x, four), from_lane(others.y, four)};
  return second ? u32x4{got.x, got.y, own.x, own.y} : u32x4{own.x, own.y, got.x, got.y};
}

template <class S>
FP4_D void dz_epilogue(const HeadTile& a, const HpTile& tile, const f32x4 (&acc)[S::QI][S::PJ]) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l16 = lane & 15, quarter = lane >> 4;
  const int unit = (lane >> 5) + (lane >> 3 & 2);
  const int wave_p = wave % S::WP, wave_q = wave / S::WP;
  const int64_t q0 = (int64_t)tile.tq * S::BQ + wave_q * (S::QI * 16);
  const int64_t left = a.g.Q - q0;
#pragma unroll
  for (int pj = 0; pj < S::PJ; pj += 2) {
    const int64_t p0 = (int64_t)tile.tp * S::BP + wave_p * (S::PJ * 16) + pj * 16;
    bool active[2];
    float shift[2];
    int64_t at[2];
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      const int64_t p = p0 + r * 16 + l16, t = p < a.g.P ? a.targets[p] : -1;
      active[r] = t >= 0 && t < a.V;
      // e^(z - lse) 2^15; nothing of a row without a target
      shift[r] = active[r] ? fmaf(-a.lse[p], LOG2E, 15.0f) : -INFINITY;
      at[r] = active[r] ? t - a.first - q0 : -1;
    }
#pragma unroll
    for (int i = 0; i < S::QI; i += 2) {
      uint32_t d[2][2][2];   // of two blocks of rows, two of columns, two pairs of columns
#pragma unroll
      for (int r = 0; r < 2; ++r)
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            float x[2];
#pragma unroll
            for (int v = 0; v < 2; ++v) {
              const int e = 2 * k + v, q = (i + u) * 16 + quarter * 4 + e;
              x[v] = __builtin_amdgcn_exp2f(fmaf(acc[i + u][pj + r][e], LOG2E, shift[r]));
              if (at[r] == q) x[v] -= DZ_SCALE;
              x[v] = active[r] && q < left ? x[v] : 0.0f;
            }
            d[r][u][k] = pack_f16(x[0], x[1]);
          }
      if (a.dz_across) {
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const int64_t col = q0 + (i + u) * 16 + quarter * 4 + (lane & 3), line = p0 + (lane & 4) * 4 + (lane & 8);
          const u32x4 eight = eight_rows(turn_four(d[0][u][0], d[0][u][1]), turn_four(d[1][u][0], d[1][u][1]));
          if (col < a.g.Q && line < a.ld_across) *reinterpret_cast<u32x4*>(a.dz_across + col * a.ld_across + line) = eight;
        }
      }
      if (!a.dz) continue;
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        const u32x4 eight = eight_columns(d[r][0][0], d[r][0][1], d[r][1][0], d[r][1][1]);
        const int64_t p = p0 + r * 16 + l16, col = q0 + i * 16 + unit * 8;
        if (col < a.ld && p < a.g.P) *reinterpret_cast<u32x4*>(a.dz + p * a.ld + col) = eight;
      }
    }
  }
}

// fp32 to [P x ldo], times a power of two, plus what is there.  Q is a multiple of 8.
template <class S>
FP4_D void f32_epilogue(const HeadTile& a, const HpTile& tile, const f32x4 (&acc)[S::QI][S::PJ], float* out, int64_t ldo, float factor) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l16 = lane & 15, quarter = lane >> 4;
  const int wave_p = wave % S::WP, wave_q = wave / S::WP;
  const int64_t q0 = (int64_t)tile.tq * S::BQ + wave_q * (S::QI * 16) + quarter * 4;
#pragma unroll
  for (int pj = 0; pj < S::PJ; ++pj) {
    const int64_t p = (int64_t)tile.tp * S::BP + wave_p * (S::PJ * 16) + pj * 16 + l16;
    if (p >= a.g.P) continue;
#pragma unroll
    for (int i = 0; i < S::QI; ++i) {
      const int64_t col = q0 + i * 16;
      if (col < a.g.Q) {
        f32x4* const o = reinterpret_cast<f32x4*>(out + p * ldo + col);
        f32x4 y = acc[i][pj] * factor;
        if (a.add) y += *o;
        *o = y;
      }
    }
  }
}
template <class S>
FP4_D void bf16_epilogue(const HeadTile& a, const HpTile& tile, const f32x4 (&acc)[S::QI][S::PJ], float factor) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l16 = lane & 15;
  const int unit = (lane >> 5) + (lane >> 3 & 2);
  const int wave_p = wave % S::WP, wave_q = wave / S::WP;
  const int64_t q0 = (int64_t)tile.tq * S::BQ + wave_q * (S::QI * 16) + unit * 8;
  uint16_t* const out = reinterpret_cast<uint16_t*>(a.out);
#pragma unroll
  for (int pj = 0; pj < S::PJ; ++pj) {
    const int64_t p = (int64_t)tile.tp * S::BP + wave_p * (S::PJ * 16) + pj * 16 + l16;
#pragma unroll
    for (int i = 0; i < S::QI; i += 2) {
      const f32x4 x = acc[i][pj] * factor, y = acc[i + 1][pj] * factor;
      const u32x4 eight = eight_columns(hp_pack_bf16(x.x, x.y), hp_pack_bf16(x.z, x.w), hp_pack_bf16(y.x, y.y), hp_pack_bf16(y.z, y.w));
      const int64_t col = q0 + i * 16;
      if (p < a.g.P && col < a.g.Q) *reinterpret_cast<u32x4*>(out + p * a.ld + col) = eight;
    }
  }
}

// Whether a row counts: without weights all do, otherwise those that have a target.
FP4_D bool row_counts(const float* weight, const int64_t* targets, int64_t V, int64_t row) {
  if (!weight) return true;
  const int64_t t = targets[row];
  return t >= 0 && t < V;
}
FP4_D float row_weight(const float* weight, const int64_t* targets, int64_t V, int64_t row) {
  return !row_counts(weight, targets, V, row) ? 0.0f : weight ? weight[row] : 1.0f;
}
FP4_D uint32_t pk_max_u16(uint32_t a, uint32_t b) {
  typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, a), __builtin_bit_cast(u16x2, b)));
}

// Largest magnitudes of both operands, x's under its rows' weights, from the fragments that pass anyway, in one tile of each column of tiles (w)
// and of each row (x): along the diagonal, since such tiles take longer and an XCD has whole rows of tiles.  (In launches of their own they took 50 us
// a piece of 134 MB.)  A maximum does not depend on the order of its atomics, of which there are few: they come one after another.
template <class S>
struct Largest {
  bool of_w, of_x;
  uint32_t w = 0, x[S::PJ];   // two bf16's magnitudes each
  static FP4_D bool w_here(const HeadTile& a, const HpTile& tile) { return a.amax_w && tile.tq % a.g.tiles_p == tile.tp; }
  static FP4_D bool x_here(const HeadTile& a, const HpTile& tile) { return a.amax_x && tile.tp % a.g.tiles_q == tile.tq; }
  FP4_D Largest(const HeadTile& a, const HpTile& tile) {
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    of_w = w_here(a, tile) && wave % S::WP == 0;
    of_x = x_here(a, tile) && wave / S::WP == 0;
#pragma unroll
    for (int j = 0; j < S::PJ; ++j) x[j] = 0;
  }
  FP4_D void operator()(const u32x4 (&fl)[S::PJ], const u32x4 (&fr)[S::QI]) {
    if (of_w) {
#pragma unroll
      for (int j = 0; j < S::QI; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) w = pk_max_u16(w, fr[j][i] & 0x7fff7fffu);
    }
    if (of_x) {
#pragma unroll
      for (int j = 0; j < S::PJ; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) x[j] = pk_max_u16(x[j], fl[j][i] & 0x7fff7fffu);
    }
  }
  static FP4_D uint32_t wider(uint32_t two) { return max(two << 16, two & 0xffff0000u); }
  static FP4_D void leave(uint32_t best, uint32_t* to) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) best = max(best, (uint32_t)__shfl_xor((int)best, o));
    if ((threadIdx.x & 63) == 0 && best) atomicMax(to, best);
  }
  FP4_D void leave(const HeadTile& a, const HpTile& tile) const {
    if (of_w) leave(wider(w), a.amax_w);
    if (of_x) {
      const int wave_p = (threadIdx.x >> 6) % S::WP, l16 = threadIdx.x & 15;
      uint32_t best = 0;
#pragma unroll
      for (int j = 0; j < S::PJ; ++j) {   // rows behind the edge repeat the last one
        const int64_t p = min((int64_t)tile.tp * S::BP + wave_p * (S::PJ * 16) + j * 16 + l16, a.g.P - 1);
        const int64_t t = a.targets[p];
        if (t >= 0 && t < a.V) best = max(best, f2u(u2f(wider(x[j])) * fabsf(a.dloss[p])));   // a row that does not count may hold anything
      }
      leave(best, a.amax_x);
    }
  }
};

// A tile of logits or of a gradient product.  256 x 256, measured: 8192 x 32000 over 2048 (maxima and sums) 0.81 ms, 1.33e15 operations/s; 32768 x 4096 over 8192 (dw) 1.56 ms,
// 1.41e15; dz's tiles end with 128 KB of stores twice, 1.2e15 over 4096, 0.64e15 over 1376.  Bound by power: in long runs the clock falls to 1.6 GHz, the matrix
// cores are busy in 52 - 68 % of the cycles, LDS conflicts are none.  Two waves a SIMD: without that bound the compiler takes 512 registers for the
// 128 x 128 tile and moves every fragment through accumulation registers.
// Tried: waves of 128 x 128 sums, one a SIMD: at a lower clock and no faster with 32 x 32 x 16 instructions; with 16 x 16 x 32 ones they do not fit their registers.
template <class S, int EPI>
__global__ __launch_bounds__(S::WAVES * 64, 2) void head_tile_kernel(HeadTile a) {
  __shared__ __attribute__((aligned(16))) uint8_t smem[S::SMEM];
  f32x4 acc[S::QI][S::PJ];
  const HpTile tile = hp_tile_at(a.g);
  if constexpr (EPI == EPI_DZ) {
    if (Largest<S>::w_here(a, tile) || Largest<S>::x_here(a, tile)) {   // the others' loop stays free of branches
      Largest<S> largest(a, tile);
      hp_tile_sums<S, false>(a.g, tile, smem, acc, largest);
      largest.leave(a, tile);
    } else {
      hp_tile_sums<S, false>(a.g, tile, smem, acc, [](const auto&, const auto&) {});
    }
  } else {
    hp_tile_sums<S, EPI != EPI_STATS>(a.g, tile, smem, acc, [](const auto&, const auto&) {});
  }
  if constexpr (EPI == EPI_STATS) stats_epilogue<S>(a, tile, smem, acc);
  if constexpr (EPI == EPI_DZ) dz_epilogue<S>(a, tile, acc);
  if constexpr (EPI == EPI_ADD) f32_epilogue<S>(a, tile, acc, a.sums + (int64_t)tile.split * a.g.P * a.g.Q, a.g.Q, scale_of(*a.amax, true) / DZ_SCALE);
  if constexpr (EPI == EPI_OUT) {
    const float factor = scale_of(*a.amax, true) / DZ_SCALE;
    if (a.out_bf16) bf16_epilogue<S>(a, tile, acc, factor);
    else f32_epilogue<S>(a, tile, acc, reinterpret_cast<float*>(a.out), a.ld, factor);
  }
}

// The tiles' maxima and sums of ROWS rows, each 1024 / ROWS-th of them by one thread, joined in order.
template <int ROWS>
__global__ __launch_bounds__(1024) void head_join_kernel(const float2* part, int tiles, int64_t M, int64_t V, const int64_t* targets, const float* target_z,
                                                         float* loss, float* lse) {
  constexpr int SHARES = 1024 / ROWS, AT_ONCE = 4;
  __shared__ float2 lds[SHARES][ROWS];
  const int r = threadIdx.x % ROWS, k = threadIdx.x / ROWS;
  const int64_t p = (int64_t)blockIdx.x * ROWS + r, row = min(p, M - 1);
  float m = -INFINITY, s = 0.0f;
  const auto join = [&](float2 o) {
    if (o.y != 0.0f) {
      const float top = fmaxf(m, o.x);
      s = s * (m == top ? 1.0f : __builtin_amdgcn_exp2f((m - top) * LOG2E)) + o.y * (o.x == top ? 1.0f : __builtin_amdgcn_exp2f((o.x - top) * LOG2E));
      m = top;
    }
  };
  for (int i0 = k; i0 < tiles; i0 += SHARES * AT_ONCE) {
    float2 o[AT_ONCE];
#pragma unroll
    for (int u = 0; u < AT_ONCE; ++u) o[u] = part[(int64_t)min(i0 + u * SHARES, tiles - 1) * M + row];
#pragma unroll
    for (int u = 0; u < AT_ONCE; ++u)
      if (i0 + u * SHARES < tiles) join(o[u]);
  }
  lds[k][r] = float2{m, s};
  for (int half = SHARES / 2; half > 0; half /= 2) {
    __syncthreads();
    if (k < half) {
      m = lds[k][r].x;
      s = lds[k][r].y;
      join(lds[k + half][r]);
      lds[k][r] = float2{m, s};
    }
  }
  if (k || p >= M) return;
  const float l = m + logf(s);
  if (lse) lse[p] = l;
  const int64_t t = targets[p];
  if (loss) loss[p] = t >= 0 && t < V ? l - target_z[p] : 0.0f;
}

__global__ __launch_bounds__(256) void clear_words_kernel(uint32_t* x, int n) {
  for (int i = threadIdx.x; i < n; i += 256) x[i] = 0;
}

// A matrix that is transposed into fp16 under a power of two: bf16 x [rows x cols], cols a multiple of 8, rows under a weight of their own where there
// are any -> out [cols x pitch], pitch a multiple of 64, zeros from rows on.
struct Across {
  const uint16_t* x;
  int64_t rows, cols, ld;
  uint16_t* out;
  int64_t pitch;
  const uint32_t* amax;      // bits of the largest magnitude
  const float* weight;
  const int64_t* targets;
  int64_t V;
};
struct AcrossBoth { Across m[2]; int groups; };   // workgroups of the first

// 134 MB in 36 - 54 us, as what the launch before wrote still leaves the last-level cache.  64 x 64 a wave: a lane turns eight rows of eight columns in its registers, of which both its loads and its stores are whole 128-byte lines of eight
// lanes each.
__global__ __launch_bounds__(256) void head_across_kernel(AcrossBoth both) {
  const bool second = (int)blockIdx.x >= both.groups;
  const Across& a = both.m[second];
  const int64_t lines = a.pitch / 64, tile = (int64_t)(second ? blockIdx.x - both.groups : blockIdx.x) * 4 + (threadIdx.x >> 6);
  const int64_t r0 = tile % lines * 64 + (threadIdx.x >> 3 & 7) * 8, c0 = tile / lines * 64 + (threadIdx.x & 7) * 8;
  if (c0 >= a.cols) return;
  const float scale = scale_of(*a.amax, false);
  u32x4 w[8];
#pragma unroll
  for (int k = 0; k < 8; ++k) w[k] = *reinterpret_cast<const u32x4*>(a.x + min(r0 + k, a.rows - 1) * a.ld + c0);
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    const bool counts = r0 + k < a.rows && row_counts(a.weight, a.targets, a.V, r0 + k);   // zeros of the others, whatever they hold
    const float f = counts && a.weight ? a.weight[r0 + k] : 1.0f;
#pragma unroll
    for (int i = 0; i < 4; ++i) w[k][i] = counts ? pack_f16(u2f(w[k][i] << 16) * f * scale, u2f(w[k][i] & 0xffff0000u) * f * scale) : 0u;
  }
#pragma unroll
  for (int c = 0; c < 8; ++c) {
    u32x4 t;
#pragma unroll
    for (int k = 0; k < 4; ++k) t[k] = __builtin_amdgcn_perm(w[2 * k + 1][c / 2], w[2 * k][c / 2], c % 2 ? 0x07060302u : 0x05040100u);
    *reinterpret_cast<u32x4*>(a.out + (c0 + c) * a.pitch + r0) = t;
  }
}

// dx's sums for few tokens, w read as it lies, once for up to 64 of them and by two workgroups for more: 256 columns a workgroup, whose four waves share a part of the vocabulary.  A lane loads eight
// rows of eight columns and turns them in its registers into eight operands, each eight rows of one column (matrix instruction f
// takes columns 8 n + f), so that nothing passes through LDS.  w stays bf16; dz's 11 bits are the sum of two bf16, a product each: it is w's bytes that bound this
// (131072 x 4096 for one token 175 us, 6.1 TB/s).
struct FewDx {
  const uint16_t *dz, *w;
  float* sums;               // [splits][M x D]
  int64_t M, D, ld, ldw, rows;   // rows: of w, dz has zeros behind them
  int64_t share;             // rows of a split, a multiple of 64
};
template <int PB>
__global__ __launch_bounds__(256, PB == 1 ? 2 : 1) void head_dx_few_kernel(FewDx a) {
  __shared__ __attribute__((aligned(16))) float lds[PB * 32][256];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l32 = lane & 31, h = lane >> 5;
  const int64_t m0 = (int64_t)blockIdx.z * (PB * 32), d0 = (int64_t)blockIdx.x * 256;
  const int64_t from = blockIdx.y * a.share + wave * (a.share / 4), to = min(a.ld, from + a.share / 4);
  const uint16_t* const w = a.w + min(d0 + l32 * 8, a.D - 8);
  const uint16_t* z[PB];
#pragma unroll
  for (int b = 0; b < PB; ++b) z[b] = a.dz + min(m0 + b * 32 + l32, a.M - 1) * a.ld + 8 * h;
  hp_f32x16 acc[PB][8];
#pragma unroll
  for (int b = 0; b < PB; ++b)
#pragma unroll
    for (int f = 0; f < 8; ++f)
#pragma unroll
      for (int v = 0; v < 16; ++v) acc[b][f][v] = 0.0f;
  struct Step { u32x4 w[8], z[PB]; };
  const auto load = [&](Step& s, int64_t v) {
#pragma unroll
    for (int j = 0; j < 8; ++j) s.w[j] = *reinterpret_cast<const u32x4*>(w + min(v + 8 * h + j, a.rows - 1) * a.ldw);
#pragma unroll
    for (int b = 0; b < PB; ++b) s.z[b] = *reinterpret_cast<const u32x4*>(z[b] + v);
  };
  Step next;
  if (from < to) load(next, from);
  for (int64_t v = from; v < to; v += 16) {
    const Step s = next;
    load(next, min(v + 16, to - 16));
    u32x4 high[PB], low[PB];
#pragma unroll
    for (int b = 0; b < PB; ++b)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t two = s.z[b][i];
        const hp_f16x2 x = __builtin_bit_cast(hp_f16x2, two);
        const float x0 = (float)x.x, x1 = (float)x.y;
        high[b][i] = hp_pack_bf16(x0, x1);
        low[b][i] = hp_pack_bf16(x0 - u2f(high[b][i] << 16), x1 - u2f(high[b][i] & 0xffff0000u));
      }
#pragma unroll
    for (int f = 0; f < 8; ++f) {
      u32x4 t;
#pragma unroll
      for (int j = 0; j < 4; ++j) t[j] = __builtin_amdgcn_perm(s.w[2 * j + 1][f / 2], s.w[2 * j][f / 2], f % 2 ? 0x07060302u : 0x05040100u);
#pragma unroll
      for (int b = 0; b < PB; ++b) {
        acc[b][f] = hp_mfma32(high[b], t, acc[b][f]);
        acc[b][f] = hp_mfma32(low[b], t, acc[b][f]);
      }
    }
  }
  // The waves' sums in their order.  Register 4 b + e: row 8 b + 4 h + e of the tokens, columns 8 l32 + f.
  for (int turn = 0; turn < 4; ++turn) {
    if (wave == turn) {
#pragma unroll
      for (int b = 0; b < PB; ++b)
#pragma unroll
        for (int v = 0; v < 16; ++v) {
          f32x4* const o = reinterpret_cast<f32x4*>(&lds[b * 32 + v / 4 * 8 + h * 4 + v % 4][l32 * 8]);
          f32x4 x = {acc[b][0][v], acc[b][1][v], acc[b][2][v], acc[b][3][v]}, y = {acc[b][4][v], acc[b][5][v], acc[b][6][v], acc[b][7][v]};
          if (turn > 0) {
            x += o[0];
            y += o[1];
          }
          o[0] = x;
          o[1] = y;
        }
    }
    __syncthreads();
  }
  float* const out = a.sums + (int64_t)blockIdx.y * a.M * a.D;
  for (int i = threadIdx.x; i < PB * 32 * 64; i += 256) {
    const int64_t m = m0 + i / 64, d = d0 + i % 64 * 4;
    if (m >= a.M || d >= a.D) continue;
    *reinterpret_cast<f32x4*>(out + m * a.D + d) = *reinterpret_cast<const f32x4*>(&lds[i / 64][i % 64 * 4]) * (1.0f / DZ_SCALE);
  }
}

// dx[t] = c_t sum over the splits of sums[., t], rounded to bf16.  D a multiple of 8.
__global__ __launch_bounds__(256) void head_dx_kernel(const float* sums, int splits, int64_t M, int64_t D, const float* dloss, const int64_t* targets, int64_t V,
                                                      uint16_t* dx, int64_t ld) {
  constexpr int AT_ONCE = 8;
  const int64_t n = D / 4;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < M * n; i += (int64_t)gridDim.x * 256) {
    const int64_t row = M * n >> 32 ? i / n : (uint32_t)i / (uint32_t)n, c = (i - row * n) * 4;
    const float f = row_weight(dloss, targets, V, row);
    f32x4 s = {0, 0, 0, 0};
    const auto at = [&](int k) { return *reinterpret_cast<const f32x4*>(sums + ((int64_t)k * M + row) * D + c); };
    int k0 = 0;
    for (; k0 + AT_ONCE <= splits; k0 += AT_ONCE) {
      f32x4 r[AT_ONCE];
#pragma unroll
      for (int k = 0; k < AT_ONCE; ++k) r[k] = at(k0 + k);
#pragma unroll
      for (int k = 0; k < AT_ONCE; ++k) s += r[k];
    }
    for (; k0 < splits; ++k0) s += at(k0);
    s = f == 0.0f ? f32x4{0, 0, 0, 0} : s * f;
    *reinterpret_cast<u32x2*>(dx + row * ld + c) = u32x2{hp_pack_bf16(s.x, s.y), hp_pack_bf16(s.z, s.w)};
  }
}

constexpr int64_t PIECE = int64_t{1} << 28;   // elements of dz, and of w's transposed piece
// Few tokens: their dx needs no transposed piece of w (both gradients, 4096 into 32000: 1 token 364 us with it, 213 without, 120 tokens 404 / 304).
constexpr int64_t FEW_TOKENS = 128;
static_assert(FEW_TOKENS * HP_MAX_DIM <= PIECE, "their dz is one piece");
bool few_tokens(int64_t M) { return M <= FEW_TOKENS; }

// ---- which tiles ---------------------------------------------------------------------------------------------------------------
using Large = HpShape<2, 4, 8, 4, 2>;    // 256 x 256
using Middle = HpShape<2, 2, 4, 4, 2>;   // 128 x 128, two a CU
using Few = HpShape<1, 4, 4, 2, 3>;      // 64 x 128, two a CU
using Fewest = HpShape<1, 4, 2, 2, 4>;   // 32 x 128, two a CU
constexpr int64_t LEAST_BQ = 128;

enum { TILE_LARGE, TILE_MIDDLE, TILE_FEW, TILE_FEWEST };
struct Cut { int tile, splits; };

// Few rows: the tiles that do not calculate much in vain, all of them waiting for w (64 x 32768 over 4096: 64 / 128 / 256 rows a tile 40 / 57 / 84 us;
// 128 rows 55 / 59 / 85).  More: by rounds of the chip's workgroups, in hundredths of a us (measured): a step of 64 takes a 256 x 256 tile 1.1, 1.25,
// 1.5 and 1.8 with a quarter, half, three quarters and all of the CUs at work (power) and 1.6 over several rounds, which do not keep step; two
// 128 x 128 tiles of one CU take 1.05, a single one about 0.63; a tile's start and end
// 6 and 4.  A round that is full is charged 1.6 also where it is the only one: 128 x 128 tiles then mostly need two and lose against either.  Splitting the
// contraction (only where the sums can be added up later: most > 1) brings rounds and takes sums' bytes.  dx's gradient calls, by the rule and by the best of both
// tiles under 1 to 16 splits: 200 x 4096 into 32000 292 / 291 us, 512 x 2048 into 32000 206 / 205, 1055 x 1376 into 50003 418 / 409, 1024 x 4096 into 32000 558 / 557,
// 2048 x 5120 into 32000 1245 / 1234, 4096 x 4096 into 32000 1735 / 1726; without splits the first four take 605, 493, 857 and 755.
Cut cut_of(int64_t P, int64_t Q, int64_t K, int most) {
  const int64_t steps = (K + 63) / 64;
  const auto tiles = [&](int64_t bp, int64_t bq) { return ((P + bp - 1) / bp) * ((Q + bq - 1) / bq); };
  most = (int)std::max<int64_t>(1, std::min<int64_t>(most, steps / 4));
  if (P <= FEW_TOKENS) return {P <= 32 ? TILE_FEWEST : TILE_FEW, 1};
  Cut best = {TILE_LARGE, 1};
  int64_t least = INT64_MAX;
  for (int s = 1; s <= most; ++s) {
    const int64_t k = (steps + s - 1) / s, sums = s > 1 ? s * P * Q / 10000 : 0;   // 5 bytes at 5 TB/s each: they are read again, their stores overlap
    const int64_t nl = tiles(256, 256) * s, nm = tiles(128, 128) * s, rl = nl % 256, rm = nm % 512;
    const int64_t large = nl / 256 * (160 * k + 600) + (rl ? (100 + 75 * rl / 256) * k + 600 : 0) + sums;
    const int64_t middle = nm / 512 * (105 * k + 400) + (rm ? (rm > 256 ? 105 : 63) * k + 400 : 0) + sums;
    if (large < least) least = large, best = {TILE_LARGE, s};
    if (middle < least) least = middle, best = {TILE_MIDDLE, s};
  }
  return best;
}

template <class S, int EPI>
int launch(HeadTile& a, hipStream_t s) {
  a.g.tiles_p = (int)((a.g.P + S::BP - 1) / S::BP);
  a.g.tiles_q = (int)((a.g.Q + S::BQ - 1) / S::BQ);
  head_tile_kernel<S, EPI><<<(unsigned)(a.g.tiles_p * a.g.tiles_q * a.g.splits), S::WAVES * 64, 0, s>>>(a);
  FP4_CHECK_LAUNCH();
  return FP4_OK;
}
template <int EPI>
int launch(HeadTile& a, const Cut& cut, hipStream_t s) {
  const int64_t steps = (a.g.K + 63) / 64;
  a.g.splits = cut.splits;
  a.g.split_steps = (int)((steps + cut.splits - 1) / cut.splits);
  if (cut.tile == TILE_LARGE) return launch<Large, EPI>(a, s);
  if constexpr (EPI != EPI_ADD) {   // few tokens' dx is another kernel's
    if (cut.tile == TILE_FEW) return launch<Few, EPI>(a, s);
    if (cut.tile == TILE_FEWEST) return launch<Fewest, EPI>(a, s);
  }
  return launch<Middle, EPI>(a, s);
}
template <int EPI>
int launch(HeadTile& a, hipStream_t s) { return launch<EPI>(a, cut_of(a.g.P, a.g.Q, a.g.K, 1), s); }

// ---- sizes of the pieces and of what they need -----------------------------------------------------------------------------------
int64_t up(int64_t x, int64_t a) { return (x + a - 1) / a * a; }

// Rows of w a piece: as many as the room allows, the pieces alike.
int64_t piece_rows(int64_t M, int64_t D, int64_t V) {
  const int64_t most = std::max<int64_t>(256, PIECE / (few_tokens(M) ? std::max<int64_t>(64, up(M, 64)) : std::max(up(M, 64), D)) / 256 * 256);
  const int64_t pieces = (V + most - 1) / most;
  return std::min(up((V + pieces - 1) / pieces, 256), up(V, 64));
}
size_t piece_room(int64_t lines, int64_t V) { return (size_t)std::min(lines * up(V, 64), PIECE + lines * 256) * 2; }   // never less for more lines

// Parts of dx's contraction: at most 64, within 2^25 sums.
int most_splits(int64_t M, int64_t D) { return (int)std::max<int64_t>(1, std::min<int64_t>(64, (int64_t{1} << 25) / std::max<int64_t>(1, M * D))); }
size_t sums_room(int64_t M, int64_t D) { return (size_t)std::max(M * D, std::min(64 * M * D, int64_t{1} << 25)) * 4; }

}  // namespace

// The forward pass goes over the tokens so many at a time, which bounds the tiles' maxima and sums.
constexpr int64_t FWD_TOKENS = 32768;

size_t hp_head_fwd_room(int64_t M, int64_t V) {
  M = std::min(M, FWD_TOKENS);
  return align_up((size_t)((V + LEAST_BQ - 1) / LEAST_BQ) * (size_t)M * 8, 256) + align_up((size_t)M * 4, 256) + 256;
}
size_t hp_head_bwd_room(int64_t M, int64_t D, int64_t V) {
  const int64_t Mp = up(M, 64);
  return 2 * align_up(piece_room(Mp, V), 256) + align_up(piece_room(D, V), 256) + align_up((size_t)D * Mp * 2, 256) + align_up(sums_room(M, D), 256) +
         align_up((size_t)(V / 256 + 2) * 4, 256) + 256;
}

int hp_launch_head_fwd(const uint16_t* x, const uint16_t* w, const int64_t* targets, int64_t M, int64_t D, int64_t V, int64_t ldx, int64_t ldw, float* loss,
                       float* lse, void* workspace, hipStream_t s) {
  uint8_t* room = (uint8_t*)align_up((size_t)(uintptr_t)workspace, 256);
  for (int64_t first = 0; first < M; first += FWD_TOKENS) {
    const int64_t m = std::min(FWD_TOKENS, M - first);
    const int64_t* const t = targets + first;
    HeadTile a = {};
    a.g = {x + first * ldx, w, m, V, D, ldx, ldw, 0, 0, 1, 0};
    a.targets = t;
    a.V = V;
    a.target_z = (float*)room;
    a.part = (float2*)(room + align_up((size_t)m * 4, 256));
    const int rc = launch<EPI_STATS>(a, s);
    if (rc) return rc;
    float *const to_loss = loss ? loss + first : nullptr, *const to_lse = lse ? lse + first : nullptr;
    if (m <= 256) head_join_kernel<4><<<(unsigned)((m + 3) / 4), 1024, 0, s>>>(a.part, a.g.tiles_q, m, V, t, a.target_z, to_loss, to_lse);
    else head_join_kernel<16><<<(unsigned)((m + 15) / 16), 1024, 0, s>>>(a.part, a.g.tiles_q, m, V, t, a.target_z, to_loss, to_lse);
    FP4_CHECK_LAUNCH();
  }
  return FP4_OK;
}

int hp_launch_head_bwd(const uint16_t* x, const uint16_t* w, const int64_t* targets, const float* lse, const float* dloss, int64_t M, int64_t D, int64_t V,
                       int64_t ldx, int64_t ldw, uint16_t* dx, int64_t ld_dx, void* dw, int dw_bf16, int64_t ld_dw, int accumulate, void* workspace,
                       hipStream_t s) {
  const int64_t Mp = up(M, 64), piece = piece_rows(M, D, V);
  uint8_t* at = (uint8_t*)align_up((size_t)(uintptr_t)workspace, 256);
  const auto take = [&](size_t n) {
    uint8_t* r = at;
    at += align_up(n, 256);
    return r;
  };
  const int pieces = (int)((V + piece - 1) / piece);
  uint32_t* const amax = (uint32_t*)take((size_t)(pieces + 1) * 4);   // of each piece of w; behind them of c x
  uint16_t* const dz = (uint16_t*)take(piece_room(Mp, V));
  uint16_t* const dz_across = (uint16_t*)take(piece_room(Mp, V));
  uint16_t* const w_across = (uint16_t*)take(piece_room(D, V));
  uint16_t* const x_across = (uint16_t*)take((size_t)D * Mp * 2);
  float* const sums = (float*)take(sums_room(M, D));
  // One or two matrices' transposes under the powers of two that suit them.
  const auto across = [&](const Across& first, const Across* second) {
    const auto tiles = [](const Across& a) { return (int)((a.pitch / 64 * ((a.cols + 63) / 64) + 3) / 4); };
    const AcrossBoth both = {{first, second ? *second : first}, tiles(first)};
    head_across_kernel<<<both.groups + (second ? tiles(*second) : 0), 256, 0, s>>>(both);
  };
  int rc = FP4_OK;
  if (M == 0 && !dw) return FP4_OK;
  clear_words_kernel<<<1, 256, 0, s>>>(amax, pieces + 1);
  FP4_CHECK_LAUNCH();
  const Across cx = {x, M, D, ldx, x_across, Mp, &amax[pieces], dloss, targets, V};
  const bool few = few_tokens(M);
  Cut dx_cut = cut_of(M, D, up(piece, 64), most_splits(M, D));   // one for all pieces: they add to the same sums
  for (int i = 0; i < pieces; ++i) {
    const int64_t first = i * piece, rows = std::min(piece, V - first), ld = up(rows, 64);
    const uint16_t* const wp = w + first * ldw;
    HeadTile t = {};
    if (M > 0) {
      t.g = {x, wp, M, rows, D, ldx, ldw, 0, 0, 1, 0};
      t.targets = targets;
      t.first = first;
      t.V = V;
      t.lse = lse;
      t.dz = dx ? dz : nullptr;
      t.ld = ld;
      t.dz_across = dw ? dz_across : nullptr;
      t.ld_across = Mp;
      t.amax_w = dx && !few ? &amax[i] : nullptr;
      t.amax_x = dw && i == 0 ? &amax[pieces] : nullptr;
      t.dloss = dloss;
      if ((rc = launch<EPI_DZ>(t, s))) return rc;
      const Across piece_of_w = {wp, rows, D, ldw, w_across, ld, &amax[i], nullptr, nullptr, 0};
      if (dx && !few) across(piece_of_w, dw && i == 0 ? &cx : nullptr);
      else if (dw && i == 0) across(cx, nullptr);
    }
    if (dx && few && M > 0) {   // all of w is one piece
      const int slices = (int)((D + 255) / 256), blocks = M <= 64 ? 1 : 2;
      const int64_t most = std::min<int64_t>(most_splits(M, D), std::max(1, 512 / (slices * blocks)));
      const int64_t share = up((ld + most - 1) / most, 64);
      dx_cut.splits = (int)((ld + share - 1) / share);
      const FewDx f = {dz, wp, sums, M, D, ld, ldw, rows, share};
      const dim3 grid((unsigned)slices, (unsigned)dx_cut.splits, (unsigned)blocks);
      if (M <= 32) head_dx_few_kernel<1><<<grid, 256, 0, s>>>(f);
      else head_dx_few_kernel<2><<<grid, 256, 0, s>>>(f);
      FP4_CHECK_LAUNCH();
    }
    if (dx && !few && M > 0) {
      t = {};
      t.g = {dz, w_across, M, D, ld, ld, ld, 0, 0, 1, 0};
      t.sums = sums;
      t.add = i > 0;
      t.amax = &amax[i];
      if ((rc = launch<EPI_ADD>(t, dx_cut, s))) return rc;
    }
    if (dw) {   // without tokens sums of nothing
      t = {};
      t.g = {dz_across, x_across, rows, D, up(M, 8), Mp, Mp, 0, 0, 1, 0};   // the lines' zeros reach that far
      t.out = (uint8_t*)dw + first * ld_dw * (dw_bf16 ? 2 : 4);
      t.out_bf16 = dw_bf16 != 0;
      t.ld = ld_dw;
      t.add = accumulate != 0;
      t.amax = &amax[pieces];
      if ((rc = launch<EPI_OUT>(t, s))) return rc;
    }
  }
  if (dx && M > 0) head_dx_kernel<<<(unsigned)std::min<int64_t>((M * (D / 4) + 255) / 256, 1 << 22), 256, 0, s>>>(sums, dx_cut.splits, M, D, dloss, targets, V, dx, ld_dx);
  FP4_CHECK_LAUNCH();
  return FP4_OK;
}
