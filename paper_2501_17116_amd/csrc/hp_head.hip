// The head: logits, softmax cross entropy and its gradients, the vocabulary in pieces.
//
//   z = x w^T,  lse_t = log sum_v e^z[t, v],  loss_t = lse_t - z[t, target_t]
//   dz[t, v] = c_t (e^(z[t, v] - lse_t) - [v = target_t]),  c_t the gradient of loss_t;   dx = dz w,  dw = dz^T x
//
// Forward: tiles of z in registers, of which a tile leaves each row's maximum m and sum of e^(z - m), and the target's z; a second launch joins the tiles
// in their order.
// Backward, a piece of the vocabulary at a time: its logits again, of which e^(z - lse) - [target] is kept as fp16 under 2^15 (11 bits; its
// values lie in [-1, 1], and below 2^-29 of 1 an element loses bits, below 2^-40 all of them); dx adds the product with the piece of w, dw's rows are the product
// with c x.  Both contract over what lies across in memory, so transposed copies are made, and as they are made anyway they are made in fp16, under
// a power of two that brings their largest element to [2^14, 2^15): w's bf16 keep all their bits unless they lie 2^-31 below it, c x is rounded
// to 11 bits.  (With bf16 operands the products' error would be that of the bf16 outputs' own rounding over again.)  Sums are fp32.
#include "hp_gemm.h"

#include <algorithm>

int fp4_compute_units_of_current_device();

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
  uint16_t* dz;              // DZ: [P x ld], zeros from Q to ld
  int64_t ld;
  float* sums;               // ADD: [splits][P x Q]
  bool add;                  // ADD, OUT: to what is there
  const uint32_t* amax;      // ADD, OUT: of the operand under a power of two
  void* out;                 // OUT
  bool out_bf16;
};

template <class S>
FP4_D void stats_epilogue(const HeadTile& a, const HpTile& tile, uint8_t* smem, const hp_f32x16 (&acc)[S::QI][S::PJ]) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l32 = lane & 31, h = lane >> 5;
  const int wave_p = wave % S::WP, wave_q = wave / S::WP;
  const int64_t q0 = (int64_t)tile.tq * S::BQ + wave_q * (S::QI * 32), left = a.g.Q - q0;
  float2* const lds = reinterpret_cast<float2*>(smem);   // [WQ][BP]
#pragma unroll
  for (int pj = 0; pj < S::PJ; ++pj) {
    const int row = wave_p * (S::PJ * 32) + pj * 32 + l32;
    const int64_t p = (int64_t)tile.tp * S::BP + row;
    const int64_t t = p < a.g.P ? a.targets[p] : -1;
    float m = -INFINITY;
    if (left >= S::QI * 32) {
#pragma unroll
      for (int i = 0; i < S::QI; ++i)
#pragma unroll
        for (int v = 0; v < 16; ++v) m = fmaxf(m, acc[i][pj][v]);
    } else {
#pragma unroll
      for (int i = 0; i < S::QI; ++i)
#pragma unroll
        for (int v = 0; v < 16; ++v) m = i * 32 + v / 4 * 8 + h * 4 + v % 4 < left ? fmaxf(m, acc[i][pj][v]) : m;
    }
    m = fmaxf(m, hp_other_half(m));
    const float ml = m == -INFINITY ? 0.0f : m * LOG2E;   // of nothing, or nothing finite
    float s = 0.0f;
#pragma unroll
    for (int i = 0; i < S::QI; ++i)
#pragma unroll
      for (int v = 0; v < 16; ++v) {
        const float e = __builtin_amdgcn_exp2f(fmaf(acc[i][pj][v], LOG2E, -ml));
        s += i * 32 + v / 4 * 8 + h * 4 + v % 4 < left ? e : 0.0f;
      }
    s += hp_other_half(s);
    if (h == 0) lds[wave_q * S::BP + row] = float2{m, s};
    const bool here = t >= q0 && t < q0 + std::min<int64_t>(left, S::QI * 32);
    if (__ballot(here)) {
      const int at = (int)(t - q0);
#pragma unroll
      for (int i = 0; i < S::QI; ++i)
#pragma unroll
        for (int v = 0; v < 16; ++v)
          if (here && at == i * 32 + v / 4 * 8 + h * 4 + v % 4) a.target_z[p] = acc[i][pj][v];
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
      if (o.y > 0.0f) s += o.y * __builtin_amdgcn_exp2f((o.x - m) * LOG2E);
    }
    a.part[(int64_t)tile.tq * a.g.P + p] = float2{m, s};
  }
}

FP4_D uint32_t pack_f16(float a, float b) {
  const hp_f16x2 v = {(_Float16)a, (_Float16)b};
  return __builtin_bit_cast(uint32_t, v);
}

// Sixteen sums of a 32 x 32 block as packed pairs -> two pieces of eight columns: of rows r16 and 16 + r16, columns 8 unit on, unit =
// lane / 32 + 2 (lane / 16 % 2), so that a store is 64 bytes of a row.
FP4_D void spread16(uint32_t (&d)[8]) {
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    hp_swap32(d[i], d[2 + i]);
    hp_swap32(d[4 + i], d[6 + i]);
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) hp_swap16(d[i], d[4 + i]);
}

template <class S>
FP4_D void dz_epilogue(const HeadTile& a, const HpTile& tile, const hp_f32x16 (&acc)[S::QI][S::PJ]) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l32 = lane & 31, h = lane >> 5;
  const int r16 = lane & 15, unit = (lane >> 5) + (lane >> 3 & 2);
  const int wave_p = wave % S::WP, wave_q = wave / S::WP;
  const int64_t q0 = (int64_t)tile.tq * S::BQ + wave_q * (S::QI * 32);
  const int64_t left = a.g.Q - q0;
#pragma unroll
  for (int pj = 0; pj < S::PJ; ++pj) {
    const int64_t p0 = (int64_t)tile.tp * S::BP + wave_p * (S::PJ * 32) + pj * 32, p = p0 + l32;
    const bool in = p < a.g.P;
    const int64_t t = in ? a.targets[p] : -1;
    const bool active = t >= 0 && t < a.V;
    // e^(z - lse) 2^15; nothing of a row without a target
    const float shift = active ? fmaf(-a.lse[p], LOG2E, 15.0f) : -INFINITY;
    const int64_t at = active ? t - a.first - q0 : -1;
#pragma unroll
    for (int i = 0; i < S::QI; ++i) {
      uint32_t d[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        float e[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const int v = 2 * k + u, q = i * 32 + v / 4 * 8 + h * 4 + v % 4;
          e[u] = __builtin_amdgcn_exp2f(fmaf(acc[i][pj][v], LOG2E, shift));
          if (at == q) e[u] -= DZ_SCALE;
          e[u] = active && q < left ? e[u] : 0.0f;
        }
        d[k] = pack_f16(e[0], e[1]);
      }
      spread16(d);
      const int64_t col = q0 + i * 32 + unit * 8;
      if (col < a.ld) {
        if (p0 + r16 < a.g.P) *reinterpret_cast<u32x4*>(a.dz + (p0 + r16) * a.ld + col) = u32x4{d[0], d[1], d[2], d[3]};
        if (p0 + 16 + r16 < a.g.P) *reinterpret_cast<u32x4*>(a.dz + (p0 + 16 + r16) * a.ld + col) = u32x4{d[4], d[5], d[6], d[7]};
      }
    }
  }
}

// fp32 to [P x ldo], times a power of two, plus what is there.  Q is a multiple of 8.
template <class S>
FP4_D void f32_epilogue(const HeadTile& a, const HpTile& tile, const hp_f32x16 (&acc)[S::QI][S::PJ], float* out, int64_t ldo, float factor) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int r16 = lane & 15, unit = (lane >> 5) + (lane >> 3 & 2);
  const int wave_p = wave % S::WP, wave_q = wave / S::WP;
  const int64_t q0 = (int64_t)tile.tq * S::BQ + wave_q * (S::QI * 32);
#pragma unroll
  for (int pj = 0; pj < S::PJ; ++pj) {
    const int64_t p0 = (int64_t)tile.tp * S::BP + wave_p * (S::PJ * 32) + pj * 32;
#pragma unroll
    for (int j = 0; j < S::QI * 2; ++j) {   // columns 16 j + 4 unit on, of the first sixteen rows and of the others
      f32x4 y[2];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        uint32_t u = f2u(acc[j / 2][pj][(j % 2) * 8 + i]), w = f2u(acc[j / 2][pj][(j % 2) * 8 + 4 + i]);
        hp_swap16(u, w);
        y[0][i] = u2f(u) * factor;
        y[1][i] = u2f(w) * factor;
      }
      const int64_t col = q0 + 16 * j + 4 * unit;
#pragma unroll
      for (int v = 0; v < 2; ++v) {
        const int64_t p = p0 + 16 * v + r16;
        if (p < a.g.P && col < a.g.Q) {
          f32x4* const o = reinterpret_cast<f32x4*>(out + p * ldo + col);
          if (a.add) y[v] += *o;
          *o = y[v];
        }
      }
    }
  }
}
template <class S>
FP4_D void bf16_epilogue(const HeadTile& a, const HpTile& tile, const hp_f32x16 (&acc)[S::QI][S::PJ], float factor) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int r16 = lane & 15, unit = (lane >> 5) + (lane >> 3 & 2);
  const int wave_p = wave % S::WP, wave_q = wave / S::WP;
  const int64_t q0 = (int64_t)tile.tq * S::BQ + wave_q * (S::QI * 32);
  uint16_t* const out = reinterpret_cast<uint16_t*>(a.out);
#pragma unroll
  for (int pj = 0; pj < S::PJ; ++pj) {
    const int64_t p0 = (int64_t)tile.tp * S::BP + wave_p * (S::PJ * 32) + pj * 32;
#pragma unroll
    for (int i = 0; i < S::QI; ++i) {
      uint32_t d[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) d[k] = hp_pack_bf16(acc[i][pj][2 * k] * factor, acc[i][pj][2 * k + 1] * factor);
      spread16(d);
      const int64_t col = q0 + i * 32 + unit * 8;
      if (col < a.g.Q) {
        if (p0 + r16 < a.g.P) *reinterpret_cast<u32x4*>(out + (p0 + r16) * a.ld + col) = u32x4{d[0], d[1], d[2], d[3]};
        if (p0 + 16 + r16 < a.g.P) *reinterpret_cast<u32x4*>(out + (p0 + 16 + r16) * a.ld + col) = u32x4{d[4], d[5], d[6], d[7]};
      }
    }
  }
}

template <class S, int EPI>
__global__ __launch_bounds__(S::WAVES * 64) void head_tile_kernel(HeadTile a) {
  __shared__ __attribute__((aligned(16))) uint8_t smem[S::SMEM];
  hp_f32x16 acc[S::QI][S::PJ];
  const HpTile tile = hp_tile_at(a.g);
  hp_tile_sums<S, EPI == EPI_ADD || EPI == EPI_OUT>(a.g, tile, smem, acc);
  if constexpr (EPI == EPI_STATS) stats_epilogue<S>(a, tile, smem, acc);
  if constexpr (EPI == EPI_DZ) dz_epilogue<S>(a, tile, acc);
  if constexpr (EPI == EPI_ADD) f32_epilogue<S>(a, tile, acc, a.sums + (int64_t)tile.split * a.g.P * a.g.Q, a.g.Q, scale_of(*a.amax, true) / DZ_SCALE);
  if constexpr (EPI == EPI_OUT) {
    const float factor = scale_of(*a.amax, true) / DZ_SCALE;
    if (a.out_bf16) bf16_epilogue<S>(a, tile, acc, factor);
    else f32_epilogue<S>(a, tile, acc, reinterpret_cast<float*>(a.out), a.ld, factor);
  }
}

// The tiles' maxima and sums of sixteen rows, each sixty-fourth of them by one thread, joined in order.
__global__ __launch_bounds__(1024) void head_join_kernel(const float2* part, int tiles, int64_t M, int64_t V, const int64_t* targets, const float* target_z,
                                                         float* loss, float* lse) {
  __shared__ float2 lds[64][16];
  const int r = threadIdx.x & 15, k = threadIdx.x >> 4;
  const int64_t p = (int64_t)blockIdx.x * 16 + r;
  float m = -INFINITY, s = 0.0f;
  const auto join = [&](float2 o) {
    const float top = fmaxf(m, o.x);
    if (o.y > 0.0f) {
      s = s * (m == top ? 1.0f : __builtin_amdgcn_exp2f((m - top) * LOG2E)) + o.y * (o.x == top ? 1.0f : __builtin_amdgcn_exp2f((o.x - top) * LOG2E));
      m = top;
    }
  };
  if (p < M)
    for (int i = k; i < tiles; i += 64) join(part[(int64_t)i * M + p]);
  lds[k][r] = float2{m, s};
  __syncthreads();
  if (k || p >= M) return;
  for (int i = 1; i < 64; ++i) join(lds[i][r]);
  const float l = m + logf(s);
  if (lse) lse[p] = l;
  const int64_t t = targets[p];
  if (loss) loss[p] = t >= 0 && t < V ? l - target_z[p] : 0.0f;
}

__global__ void clear_words_kernel(uint32_t* x, int n) {
  if ((int)threadIdx.x < n) x[threadIdx.x] = 0;
}

FP4_D float row_weight(const float* weight, const int64_t* targets, int64_t V, int64_t row) {
  if (!weight) return 1.0f;
  const int64_t t = targets[row];
  return t >= 0 && t < V ? weight[row] : 0.0f;
}

// Largest magnitude of bf16 x [rows x cols], rows under a weight of their own where there are any; bits of the fp32 value.  A maximum does not depend on
// the order of its atomics.  cols a multiple of 8.
__global__ __launch_bounds__(256) void head_amax_kernel(const uint16_t* x, int64_t rows, int64_t cols, int64_t ld, const float* weight, const int64_t* targets,
                                                        int64_t V, uint32_t* amax) {
  uint32_t best = 0;
  for (int64_t r = blockIdx.x; r < rows; r += gridDim.x) {
    uint32_t m = 0;
    for (int64_t c = (int64_t)threadIdx.x * 8; c < cols; c += 2048) {
      const u32x4 w = *reinterpret_cast<const u32x4*>(x + r * ld + c);
#pragma unroll
      for (int i = 0; i < 4; ++i) m = max(m, max(w[i] << 16 & 0x7fffffffu, w[i] & 0x7fff0000u));
    }
    best = max(best, f2u(u2f(m) * fabsf(row_weight(weight, targets, V, r))));
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) best = max(best, (uint32_t)__shfl_xor((int)best, o));
  if ((threadIdx.x & 63) == 0 && best) atomicMax(amax, best);
}

// x [rows x cols] -> its transpose in fp16 [cols x pitch], zeros from rows to pitch.  x: bf16, under a power of two and rows' weights, or
// (F16) fp16 as it is.  64 x 64 a workgroup, through LDS; pitch a multiple of 64.
struct Across {
  const uint16_t* x;
  int64_t rows, cols, ld;
  uint16_t* out;
  int64_t pitch;
  const uint32_t* amax;
  const float* weight;
  const int64_t* targets;
  int64_t V;
};
template <bool F16>
__global__ __launch_bounds__(256) void head_across_kernel(Across a) {
  __shared__ uint16_t lds[64][66];
  const int64_t r0 = (int64_t)blockIdx.x * 64, c0 = (int64_t)blockIdx.y * 64;
  const int chunk = threadIdx.x & 7;
  const float scale = F16 ? 1.0f : scale_of(*a.amax, false);
#pragma unroll
  for (int half = 0; half < 2; ++half) {
    const int r = half * 32 + (threadIdx.x >> 3);
    const int64_t row = r0 + r, col = c0 + chunk * 8;
    u32x4 w = {0, 0, 0, 0};
    if (row < a.rows && col < a.cols) {
      w = *reinterpret_cast<const u32x4*>(a.x + row * a.ld + col);
      if constexpr (!F16) {
        const float f = row_weight(a.weight, a.targets, a.V, row);
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = pack_f16(u2f(w[i] << 16) * f * scale, u2f(w[i] & 0xffff0000u) * f * scale);
      }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) *reinterpret_cast<uint32_t*>(&lds[r][chunk * 8 + 2 * i]) = w[i];
  }
  __syncthreads();
#pragma unroll
  for (int half = 0; half < 2; ++half) {
    const int c = half * 32 + (threadIdx.x >> 3);
    const int64_t col = c0 + c, row = r0 + chunk * 8;
    if (col >= a.cols) continue;
    u32x4 w;
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = lds[chunk * 8 + 2 * i][c] | (uint32_t)lds[chunk * 8 + 2 * i + 1][c] << 16;
    *reinterpret_cast<u32x4*>(a.out + col * a.pitch + row) = w;
  }
}

// dx[t] = c_t sum over the splits of sums[., t], rounded to bf16.  D a multiple of 8.
__global__ __launch_bounds__(256) void head_dx_kernel(const float* sums, int splits, int64_t M, int64_t D, const float* dloss, const int64_t* targets, int64_t V,
                                                      uint16_t* dx, int64_t ld) {
  const int64_t n = D / 8, i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= M * n) return;
  const int64_t row = i / n, c = i % n * 8;
  const float f = row_weight(dloss, targets, V, row);
  float s[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) s[e] = 0.0f;
  for (int k = 0; k < splits; ++k) {
    const Raw8<F32> r = hp_load8<F32>(sums + ((int64_t)k * M + row) * D, c, D);
#pragma unroll
    for (int e = 0; e < 8; ++e) s[e] += r.get(e);
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) s[e] = f == 0.0f ? 0.0f : s[e] * f;
  hp_store8<BF16>(dx + row * ld, c, D, s);
}

// ---- which tiles ---------------------------------------------------------------------------------------------------------------
using Large = HpShape<2, 4, 4, 2, 2>;    // 256 x 256
using Middle = HpShape<2, 2, 2, 2, 3>;   // 128 x 128
using Few = HpShape<1, 4, 2, 1, 3>;      // 64 x 128
using Fewest = HpShape<1, 4, 1, 1, 4>;   // 32 x 128
constexpr int64_t LEAST_BQ = 128;

enum { TILE_LARGE, TILE_MIDDLE, TILE_FEW, TILE_FEWEST };
int tile_of(int64_t P, int64_t Q) {
  if (P <= 32) return TILE_FEWEST;
  if (P <= 64) return TILE_FEW;
  const int64_t large = ((P + 255) / 256) * ((Q + 255) / 256);
  return P <= 128 || large < 128 ? TILE_MIDDLE : TILE_LARGE;
}
void tile_size(int tile, int64_t& bp, int64_t& bq) {
  bp = tile == TILE_LARGE ? 256 : tile == TILE_MIDDLE ? 128 : tile == TILE_FEW ? 64 : 32;
  bq = tile == TILE_LARGE ? 256 : 128;
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
int launch(HeadTile& a, hipStream_t s) {
  const int tile = tile_of(a.g.P, a.g.Q);
  const int64_t steps = (a.g.K + 63) / 64;
  a.g.split_steps = (int)((steps + a.g.splits - 1) / a.g.splits);
  switch (tile) {
    case TILE_LARGE: return launch<Large, EPI>(a, s);
    case TILE_MIDDLE: return launch<Middle, EPI>(a, s);
    case TILE_FEW: return launch<Few, EPI>(a, s);
    default: return launch<Fewest, EPI>(a, s);
  }
}

// ---- sizes of the pieces and of what they need -----------------------------------------------------------------------------------
constexpr int64_t PIECE = int64_t{1} << 27;   // elements of dz, and of w's transposed piece
int64_t up(int64_t x, int64_t a) { return (x + a - 1) / a * a; }

// Rows of w a piece: as many as the room allows, the pieces alike.
int64_t piece_rows(int64_t M, int64_t D, int64_t V) {
  const int64_t most = std::max<int64_t>(256, PIECE / std::max(up(M, 64), D) / 256 * 256);
  const int64_t pieces = (V + most - 1) / most;
  return std::min(up((V + pieces - 1) / pieces, 256), up(V, 64));
}
size_t piece_room(int64_t lines, int64_t V) { return (size_t)std::min(lines * up(V, 64), PIECE + lines * 256) * 2; }   // never less for more lines

// Parts of dx's contraction: where its tiles are few, so many that the chip is full, within 2^25 sums.
int dx_splits(int64_t M, int64_t D, int64_t piece) {
  int64_t bp, bq;
  tile_size(tile_of(M, D), bp, bq);
  const int64_t tiles = ((M + bp - 1) / bp) * ((D + bq - 1) / bq), steps = (piece + 63) / 64;
  int64_t s = std::min<int64_t>(std::min<int64_t>(64, 512 / std::max<int64_t>(1, tiles)), steps / 4);
  s = std::min(s, (int64_t{1} << 25) / std::max<int64_t>(1, M * D));
  return (int)std::max<int64_t>(1, s);
}
size_t sums_room(int64_t M, int64_t D) { return (size_t)std::max(M * D, std::min(64 * M * D, int64_t{1} << 25)) * 4; }

}  // namespace

size_t hp_head_fwd_room(int64_t M, int64_t V) {
  return align_up((size_t)((V + LEAST_BQ - 1) / LEAST_BQ) * (size_t)M * 8, 256) + align_up((size_t)M * 4, 256) + 256;
}
size_t hp_head_bwd_room(int64_t M, int64_t D, int64_t V) {
  const int64_t Mp = up(M, 64);
  return 2 * align_up(piece_room(Mp, V), 256) + align_up(piece_room(D, V), 256) + align_up((size_t)D * Mp * 2, 256) + align_up(sums_room(M, D), 256) + 512;
}

int hp_launch_head_fwd(const uint16_t* x, const uint16_t* w, const int64_t* targets, int64_t M, int64_t D, int64_t V, int64_t ldx, int64_t ldw, float* loss,
                       float* lse, void* workspace, hipStream_t s) {
  uint8_t* room = (uint8_t*)align_up((size_t)(uintptr_t)workspace, 256);
  HeadTile a = {};
  a.g = {x, w, M, V, D, ldx, ldw, 0, 0, 1, 0};
  a.targets = targets;
  a.V = V;
  a.target_z = (float*)room;
  a.part = (float2*)(room + align_up((size_t)M * 4, 256));
  const int rc = launch<EPI_STATS>(a, s);
  if (rc) return rc;
  head_join_kernel<<<(unsigned)((M + 15) / 16), 1024, 0, s>>>(a.part, a.g.tiles_q, M, V, targets, a.target_z, loss, lse);
  FP4_CHECK_LAUNCH();
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
  uint32_t* const amax = (uint32_t*)take(8);   // [0]: of c x, [1]: of the piece of w
  uint16_t* const dz = (uint16_t*)take(piece_room(Mp, V));
  uint16_t* const dz_across = (uint16_t*)take(piece_room(Mp, V));
  uint16_t* const w_across = (uint16_t*)take(piece_room(D, V));
  uint16_t* const x_across = (uint16_t*)take((size_t)D * Mp * 2);
  float* const sums = (float*)take(sums_room(M, D));
  const auto across = [&](auto f16, const Across& a) {
    const dim3 grid((unsigned)(a.pitch / 64), (unsigned)((a.cols + 63) / 64));
    head_across_kernel<decltype(f16)::value><<<grid, 256, 0, s>>>(a);
  };
  const auto largest = [&](const uint16_t* m, int64_t rows, int64_t ld, const float* weight, uint32_t* to) {
    clear_words_kernel<<<1, 64, 0, s>>>(to, 1);
    head_amax_kernel<<<(unsigned)std::min<int64_t>(rows, 2048), 256, 0, s>>>(m, rows, D, ld, weight, targets, V, to);
  };
  int rc = FP4_OK;
  if (M == 0) {   // dw's rows are sums of nothing
    if (!dw) return FP4_OK;
    clear_words_kernel<<<1, 64, 0, s>>>(amax, 2);
  } else if (dw) {
    largest(x, M, ldx, dloss, &amax[0]);
    across(std::false_type{}, Across{x, M, D, ldx, x_across, Mp, &amax[0], dloss, targets, V});
    FP4_CHECK_LAUNCH();
  }
  const int splits = dx_splits(M, D, piece);
  for (int64_t first = 0; first < V; first += piece) {
    const int64_t rows = std::min(piece, V - first), ld = up(rows, 64);
    const uint16_t* const wp = w + first * ldw;
    HeadTile z = {};
    z.g = {x, wp, M, rows, D, ldx, ldw, 0, 0, 1, 0};
    z.targets = targets;
    z.first = first;
    z.V = V;
    z.lse = lse;
    z.dz = dz;
    z.ld = ld;
    if (M > 0 && (rc = launch<EPI_DZ>(z, s))) return rc;
    if (dx && M > 0) {
      largest(wp, rows, ldw, nullptr, &amax[1]);
      across(std::false_type{}, Across{wp, rows, D, ldw, w_across, ld, &amax[1], nullptr, nullptr, 0});
      HeadTile t = {};
      t.g = {dz, w_across, M, D, ld, ld, ld, 0, 0, splits, 0};
      t.sums = sums;
      t.add = first > 0;
      t.amax = &amax[1];
      if ((rc = launch<EPI_ADD>(t, s))) return rc;
    }
    if (dw) {
      if (M > 0) across(std::true_type{}, Across{dz, M, rows, ld, dz_across, Mp, nullptr, nullptr, nullptr, 0});
      HeadTile t = {};
      t.g = {dz_across, x_across, rows, D, Mp, Mp, Mp, 0, 0, 1, 0};
      t.out = (uint8_t*)dw + first * ld_dw * (dw_bf16 ? 2 : 4);
      t.out_bf16 = dw_bf16 != 0;
      t.ld = ld_dw;
      t.add = accumulate != 0;
      t.amax = &amax[0];
      if ((rc = launch<EPI_OUT>(t, s))) return rc;
    }
  }
  if (dx && M > 0) head_dx_kernel<<<(unsigned)((M * (D / 8) + 255) / 256), 256, 0, s>>>(sums, splits, M, D, dloss, targets, V, dx, ld_dx);
  FP4_CHECK_LAUNCH();
  return FP4_OK;
}
