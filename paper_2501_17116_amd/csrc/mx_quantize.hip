// Microscaled quantization along rows, along columns (transposed) and both from one read, and the way back.
//
// A block's scale depends on its 32 elements alone, so every pass reads its input once and is bound by memory: b + 1/2 + 1/32 bytes an
// element for 4 bits along one axis (b = 2 bf16, 4 fp32), b + 1 + 1/32 for 8, their sum without the second b for both axes.
//   rows: four lanes hold a block of bf16 (eight elements, 16 bytes each), so a wave takes 512 elements of a row, loads, codes and
//         scales are contiguous, and the block's maximum is two lane exchanges away.
//   columns: a wave takes 32 rows; the rows' 16-byte pieces go through the wave's own LDS and come back as one dword a row, a lane
//         holding its columns' whole blocks: maxima and codes need no exchange, and the codes leave transposed.  The same pieces make
//         the rows' blocks before they are parked, which is the whole cost of the second axis.
#include "mx_common.h"

#include <algorithm>
#include <type_traits>

int fp4_compute_units_of_current_device();

namespace {

constexpr int NO_AXIS = 0;

struct QuantArgs {
  const void* x;
  int64_t rows, cols, ld;
  uint8_t *row_codes, *row_scales, *col_codes, *col_scales;
};

// of the other four lanes of eight
FP4_D uint32_t other_quad(uint32_t v) { return (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x141, 0xf, 0xf, true); }   // mirrored in eight lanes

// ---- rows --------------------------------------------------------------------------------------------------------------------
// A wave takes 512 elements of a row at a time (a unit of the pitch), ROWS_U of them from consecutive units.  Bound by memory: 16384 x 4096 bf16 to 4
// bits 29.9 us, to 8 bits 35.2 (5.7 TB/s of what has to move); 4096 x 11008 fp32 38.0 and 40.2 (5.4, 5.7).
constexpr int ROWS_U = 4;

template <class T, int BITS>
__global__ __launch_bounds__(256) void mx_rows_kernel(QuantArgs a, int64_t units, int per_row) {
  const int lane = threadIdx.x & 63;
  const int64_t u0 = ((int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6)) * ROWS_U;
  constexpr int P = sizeof(T) == 2 ? 1 : 2;   // pieces a lane
  u32x4 w[ROWS_U][P];
  auto each = [&](bool ragged) {
    int64_t row = u0 / per_row;
    int seg = (int)(u0 - row * per_row);
#pragma unroll
    for (int i = 0; i < ROWS_U; ++i) {
#pragma unroll
      for (int p = 0; p < P; ++p) w[i][p] = mx_load_piece<T>(a.x, row, a.rows, a.cols, a.ld, (int64_t)seg * MX_PITCH + lane * 8 + p * 4, ragged);
      if (++seg == per_row) {
        seg = 0;
        ++row;
      }
    }
  };
  if (a.cols % (16 / (int)sizeof(T))) each(true);
  else each(false);
#pragma unroll
  for (int i = 0; i < ROWS_U; ++i) {
    if (u0 + i >= units) break;
    uint32_t top;
    if constexpr (P == 1) top = mx_amax_bf16(w[i][0]);
    else {
      const uint32_t t0 = mx_amax_f32(w[i][0]), t1 = mx_amax_f32(w[i][P - 1]);
      top = t0 > t1 ? t0 : t1;
    }
    const uint32_t byte = mx_scale_byte<BITS>(mx_quad_max(top));
    const float s = mx_scale_f32(byte);
    const int64_t unit = u0 + i;   // lines are pitch / 512 units long, so units are numbered as they lie
    uint32_t h, l;
    if constexpr (P == 1) mx_encode8<BITS>(w[i][0], s, h, l);
    else mx_encode8<BITS>(w[i][0], w[i][P - 1], s, h, l);
    reinterpret_cast<uint32_t*>(a.row_codes)[unit * 64 + lane] = h;
    if constexpr (BITS == 8) reinterpret_cast<uint32_t*>(a.row_codes)[(units + unit) * 64 + lane] = l;
    if ((lane & 3) == 0) a.row_scales[unit * 16 + (lane >> 2)] = (uint8_t)byte;
  }
}

// ---- columns, and rows beside them ----------------------------------------------------------------------------------------------
// A wave takes 32 rows x 256 bytes of columns, one block of every column, a workgroup eight waves' rows.  The columns' codes pass through LDS
// once more, so that they leave as whole 128-byte lines (256 rows of 4-bit codes); four waves, half lines, were slower by a seventh (4 bits)
// and a fifth (8 bits).  16384 x 4096 bf16: columns in 4 bits 35.8 us, in 8 bits 40.0, rows and columns in 4 bits 44.9, rows in 4 and columns in 8
// 49.3 (4.6 - 5.1 TB/s); 4096 x 11008 fp32, both in 4 bits 53.4 (4.3).  With one to six workgroups a CU, which load, compute and store
// together, it stays below that: bf16, both in 4 bits 2048 x 5504 14.0 us (2.5 TB/s), 8192 x 5504 37.4 (3.7), in 4 and 8 bits 8192 x 2048 18.5 (3.2).
// Bound by memory; what remains above the rows' rate are some 700 vector
// instructions a wave, which four waves a SIMD do not hide altogether.  Tensors that do not give every CU such a workgroup are one wave's chain of requests and
// instructions long; there a workgroup has two waves (1055 x 1384: rows and columns in 4 bits 5.7 us in the kernel).
// What the order of the tiles costs (GROUP_C side by side before the next rows): whole rows of tiles write one line of the output every so many
// KiB at a time, columns of tiles read rows that far apart, and either may fall on a few of the memory's channels.  16384 x 4096 bf16, columns in
// 4 bits 40.1 us with whole rows, 36.2 / 38.3 / 37.7 with 4 / 8 / 16; 8192 x 11008 51.0, 54.7 / 50.3 / 51.2; 4096 x 11008 fp32 46.4, 48.9 / 48.2 / 46.8.
constexpr int GROUP_C = 16;
constexpr int64_t NEAR_LD = 0xffffffffll / 32;   // bytes from row to row with which a tile's 32 rows stay within 2^32

template <class T, int ROW, int COL, int TW>   // TW: waves
__global__ __launch_bounds__(TW * 64) void mx_tile_kernel(QuantArgs a, int tiles_c, int64_t tiles) {
  constexpr int E = sizeof(T);
  constexpr int CW = 256 / E;        // columns a tile
  constexpr int EPP = 16 / E;        // elements of a 16-byte piece
  constexpr int NC = 4 / E;          // columns a lane
  __shared__ __attribute__((aligned(16))) uint32_t park[TW][32 * 64];
  // neighbours along a row on one XCD, whose L2 joins their parts of the rows' lines
  const int64_t per_xcd = (tiles + 7) / 8, id = (int64_t)(blockIdx.x % 8) * per_xcd + blockIdx.x / 8;
  if ((int64_t)(blockIdx.x / 8) >= per_xcd || id >= tiles) return;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  // GROUP_C tiles side by side, then the next rows of the same columns
  const int64_t tiles_r = tiles / tiles_c, in_group = tiles_r * GROUP_C, group = id / in_group, at_c = group * GROUP_C;
  const int64_t wide = min((int64_t)GROUP_C, tiles_c - at_c), tr = (id - group * in_group) / wide;
  const int64_t r0 = tr * (TW * 32) + wave * 32, c0 = (at_c + (id - group * in_group) - tr * wide) * CW;
  const int64_t row_pitch = mx_pitch_of(a.cols), col_pitch = mx_pitch_of(a.rows);
  const int piece = lane & 15, sub = lane >> 4;
  u32x4 w[8];
  // Inside: eight requests and nothing between them, with 32 bits for what lies between the tile's rows.  Rows too far apart for that go the
  // edges' way, which counts in 64.
  if (r0 + 32 <= a.rows && c0 + CW <= a.cols && a.ld <= NEAR_LD / E) {
    const uint8_t* const first = reinterpret_cast<const uint8_t*>(a.x) + (r0 * a.ld + c0) * E;
    const uint32_t step = (uint32_t)a.ld * E;
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = *reinterpret_cast<const u32x4*>(first + (i * 4 + sub) * step + piece * 16);
  } else {
    auto each = [&](bool ragged) {
#pragma unroll
      for (int i = 0; i < 8; ++i) w[i] = mx_load_piece<T>(a.x, r0 + i * 4 + sub, a.rows, a.cols, a.ld, c0 + piece * EPP, ragged);
    };
    if (r0 >= a.rows || c0 >= a.cols) {   // behind the edge: zeros up to the pitch
#pragma unroll
      for (int i = 0; i < 8; ++i) w[i] = u32x4{0u, 0u, 0u, 0u};
    } else if (a.cols % EPP) each(true);
    else each(false);
  }
  uint32_t* const mine = park[wave];
#pragma unroll
  for (int i = 0; i < 8; ++i) *reinterpret_cast<u32x4*>(mine + (i * 4 + sub) * 64 + piece * 4) = w[i];
  if constexpr (ROW != NO_AXIS) {
    uint8_t *const row_h = a.row_codes + (r0 * row_pitch + c0) / 2, *const row_s = a.row_scales + (r0 * row_pitch + c0) / MX_BLOCK;
    const uint32_t rows_here = (uint32_t)max(min(a.rows - r0, (int64_t)32), (int64_t)0);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      uint32_t top = mx_quad_max(E == 2 ? mx_amax_bf16(w[i]) : mx_amax_f32(w[i]));
      if constexpr (E == 4) {
        const uint32_t o = other_quad(top);
        top = top > o ? top : o;
      }
      const uint32_t byte = mx_scale_byte<ROW>(top);
      const float s = mx_scale_f32(byte);
      const uint32_t row = (uint32_t)(i * 4 + sub);
      if (row < rows_here) {
        uint32_t h, l;
        uint8_t *const ph = row_h + row * (uint32_t)(row_pitch / 2) + piece * (EPP / 2), *const pl = ph + a.rows * row_pitch / 2;
        if constexpr (E == 2) {
          mx_encode8<ROW>(w[i], s, h, l);
          *reinterpret_cast<uint32_t*>(ph) = h;
          if constexpr (ROW == 8) *reinterpret_cast<uint32_t*>(pl) = l;
        } else {
          h = l = 0;
          mx_pair<ROW, 0>(u2f(w[i].x), u2f(w[i].y), s, h, l);
          mx_pair<ROW, 1>(u2f(w[i].z), u2f(w[i].w), s, h, l);
          *reinterpret_cast<uint16_t*>(ph) = (uint16_t)h;
          if constexpr (ROW == 8) *reinterpret_cast<uint16_t*>(pl) = (uint16_t)l;
        }
        if (piece % (MX_BLOCK / EPP) == 0) row_s[row * (uint32_t)(row_pitch / MX_BLOCK) + piece / (MX_BLOCK / EPP)] = (uint8_t)byte;
      }
    }
  }
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  uint32_t d[32];
#pragma unroll
  for (int r = 0; r < 32; ++r) d[r] = mine[r * 64 + lane];
  u32x4 hi[NC], lo[NC];
  uint32_t bytes[NC];
  uint32_t tops = 0;   // of both columns at once where a word holds two
#pragma unroll
  for (int r = 0; r < 32; ++r) {
    if constexpr (E == 2) tops = mx_pk_max_u16(tops, d[r] & 0x7fff7fffu);
    else tops = max(tops, d[r] & 0x7fffffffu);
  }
#pragma unroll
  for (int h = 0; h < NC; ++h) {
    const uint32_t top = E == 4 ? tops : h == 0 ? tops << 16 : tops & 0xffff0000u;
    bytes[h] = mx_scale_byte<COL>(top);
    const float s = mx_scale_f32(bytes[h]);
#pragma unroll
    for (int q = 0; q < 4; ++q) {   // eight rows
      uint32_t ch, cl;
      if constexpr (E == 2) {
        u32x4 pr;   // rows 2 i and 2 i + 1 of this column
#pragma unroll
        for (int i = 0; i < 4; ++i) pr[i] = __builtin_amdgcn_perm(d[8 * q + 2 * i + 1], d[8 * q + 2 * i], h == 0 ? 0x05040100u : 0x07060302u);
        mx_encode8<COL>(pr, s, ch, cl);
      } else {
        float v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = u2f(d[8 * q + i]);
        mx_encode8<COL>(v, s, ch, cl);
      }
      hi[h][q] = ch;
      lo[h][q] = cl;
    }
  }
  // [plane][column][wave], sixteen bytes each, and the scales [column][wave], over the parked rows; a column's pieces are rotated by half
  // its number, so that lanes with one piece of neighbouring columns meet all bank groups
  __syncthreads();
  uint8_t* const out = reinterpret_cast<uint8_t*>(&park[0][0]);
  uint8_t* const out_scales = out + COL / 4 * CW * (TW * 16);
#pragma unroll
  for (int h = 0; h < NC; ++h) {
    const int c = lane * NC + h, at = c * (TW * 16) + ((wave + (c >> 1)) & (TW - 1)) * 16;
    *reinterpret_cast<u32x4*>(out + at) = hi[h];
    if constexpr (COL == 8) *reinterpret_cast<u32x4*>(out + CW * (TW * 16) + at) = lo[h];
    out_scales[c * TW + wave] = (uint8_t)bytes[h];
  }
  __syncthreads();
  const int64_t first = (c0 * col_pitch + tr * (TW * 32));
  const uint32_t cols_here = (uint32_t)min(a.cols - c0, (int64_t)CW);   // negative behind the last column: none
#pragma unroll
  for (int i = 0; i < CW / 64; ++i) {
    const uint32_t n = i * TW * 64 + threadIdx.x, c = n / TW, piece16 = n % TW;
    if (a.cols > c0 && c < cols_here) {
      uint8_t* const o = a.col_codes + first / 2 + (c * (uint64_t)(col_pitch / 2) + piece16 * 16);
#pragma unroll
      for (int p = 0; p < COL / 4; ++p)
        *reinterpret_cast<u32x4*>(o + p * (a.cols * col_pitch / 2)) = *reinterpret_cast<const u32x4*>(out + (p * CW + c) * (TW * 16) + ((piece16 + (c >> 1)) & (TW - 1)) * 16);
    }
  }
  typedef typename std::conditional<TW == 8, u32x2, uint16_t>::type Scales;   // a column's
  static_assert(TW == 8 || TW == 2, "a byte a wave");
  if (threadIdx.x < CW && c0 + threadIdx.x < a.cols)
    *reinterpret_cast<Scales*>(a.col_scales + first / MX_BLOCK + threadIdx.x * (col_pitch / MX_BLOCK)) = *reinterpret_cast<const Scales*>(out_scales + threadIdx.x * TW);
}

// ---- back ----------------------------------------------------------------------------------------------------------------------
struct DequantArgs {
  const uint8_t *codes, *scales;
  void* x;
  int64_t lines, length, ld;
};

FP4_D float decode_scale(uint32_t byte) { return u2f(byte ? byte << 23 : 0x00400000u); }   // 2^(byte - 127)

// eight codes, of 8 bits two words of them, under one scale -> eight fp32; byte 255: NaN throughout, which the scale brings
template <int BITS>
FP4_D void decode8(const uint32_t (&c)[BITS / 4], uint32_t byte, float (&o)[8]) {
  const float s = byte == 255u ? u2f(0x7fffffffu) : decode_scale(byte);
  mx_f32x2 v[4];
  v[0] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c[0], 1.0f, 0);
  v[1] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c[0], 1.0f, 1);
  v[2] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c[0], 1.0f, 2);
  v[3] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c[0], 1.0f, 3);
  if constexpr (BITS == 8) {   // joined before they are scaled: s h alone may overflow
    mx_f32x2 l[4];
    l[0] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c[1], 0.125f, 0);
    l[1] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c[1], 0.125f, 1);
    l[2] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c[1], 0.125f, 2);
    l[3] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c[1], 0.125f, 3);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[i].x += l[i].x;
      v[i].y += l[i].y;
    }
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) o[i] = v[i / 2][i & 1] * s;
}
// ... -> four pairs of bf16, exactly: s (h + l / 8) has seven bits
template <int BITS>
FP4_D void decode8(const uint32_t (&c)[BITS / 4], uint32_t byte, uint32_t (&o)[4]) {
  if constexpr (BITS == 4) {
    const float s = decode_scale(byte);
    o[0] = mx_bits(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c[0], s, 0));
    o[1] = mx_bits(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c[0], s, 1));
    o[2] = mx_bits(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c[0], s, 2));
    o[3] = mx_bits(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c[0], s, 3));
    if (byte == 255u) o[0] = o[1] = o[2] = o[3] = 0x7fff7fffu;
  } else {
    float v[8];
    decode8<BITS>(c, byte, v);
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] = __builtin_amdgcn_perm(f2u(v[2 * i + 1]), f2u(v[2 * i]), 0x07060302u);
  }
}

// Eight elements of a row from column c on; the row may end among them.
FP4_D void store8(uint16_t* p, const uint32_t (&o)[4], int64_t left) {
  if (left >= 8) {
    *reinterpret_cast<u32x4*>(p) = u32x4{o[0], o[1], o[2], o[3]};
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e < left) p[e] = (uint16_t)(o[e / 2] >> (16 * (e & 1)));
  }
}
FP4_D void store8(float* p, const float (&o)[8], int64_t left) {
  if (left >= 8) {
    *reinterpret_cast<f32x4*>(p) = f32x4{o[0], o[1], o[2], o[3]};
    *reinterpret_cast<f32x4*>(p + 4) = f32x4{o[4], o[5], o[6], o[7]};
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e < left) p[e] = o[e];
  }
}
template <class T> struct Eight;
template <> struct Eight<uint16_t> { typedef uint32_t type[4]; };
template <> struct Eight<float> { typedef float type[8]; };

// Lines as rows: a lane takes eight codes.  Bound by memory: 16384 x 4096 to bf16 from 4 bits 27.6 us, from 8 bits 33.8 (6.1 TB/s).
template <class T, int BITS>
__global__ __launch_bounds__(256) void mx_restore_rows_kernel(DequantArgs a, int64_t units, int per_line) {
  const int lane = threadIdx.x & 63;
  const int64_t u0 = ((int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6)) * ROWS_U;
  uint32_t c[ROWS_U][BITS / 4], b[ROWS_U];
#pragma unroll
  for (int i = 0; i < ROWS_U; ++i) {
    const int64_t u = u0 + i < units ? u0 + i : units - 1;
#pragma unroll
    for (int k = 0; k < BITS / 4; ++k) c[i][k] = reinterpret_cast<const uint32_t*>(a.codes)[(k * units + u) * 64 + lane];
    b[i] = a.scales[u * 16 + (lane >> 2)];
  }
  int64_t line = u0 / per_line;
  int seg = (int)(u0 - line * per_line);
#pragma unroll
  for (int i = 0; i < ROWS_U; ++i) {
    if (u0 + i >= units) break;
    const int64_t at = (int64_t)seg * MX_PITCH + lane * 8;
    if (at < a.length) {
      typename Eight<T>::type o;
      decode8<BITS>(c[i], b[i], o);
      store8(reinterpret_cast<T*>(a.x) + line * a.ld + at, o, a.length - at);
    }
    if (++seg == per_line) {
      seg = 0;
      ++line;
    }
  }
}

// Lines as columns: a workgroup takes 256 elements of 64 lines, whole 128-byte lines of codes, through LDS; then a lane eight rows of eight
// columns.  A line's words in LDS are one apart from a multiple of the banks.  Bound by memory: 16384 x 4096 to bf16 from 4 bits 28.4 us (6.0 TB/s),
// from 8 bits 44.1 (4.6), 32 where the codes were just written.
template <class T, int BITS>
__global__ __launch_bounds__(256) void mx_restore_cols_kernel(DequantArgs a, int tiles_l, int64_t tiles) {
  constexpr int LW = 33;   // words a line
  __shared__ uint32_t park[BITS / 4][64 * LW];
  // neighbours along a row of x on one XCD
  const int64_t per_xcd = (tiles + 7) / 8, id = (int64_t)(blockIdx.x % 8) * per_xcd + blockIdx.x / 8;
  if ((int64_t)(blockIdx.x / 8) >= per_xcd || id >= tiles) return;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t te = id / tiles_l, e0 = te * 256, l0 = (id - te * tiles_l) * 64;
  const int64_t pitch = mx_pitch_of(a.length);
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int n = i * 256 + threadIdx.x, line = n >> 3, piece = n & 7;
    const int64_t at = (min(l0 + line, a.lines - 1) * pitch + e0) / 2 + piece * 16;
#pragma unroll
    for (int k = 0; k < BITS / 4; ++k) {
      const u32x4 v = *reinterpret_cast<const u32x4*>(a.codes + k * (a.lines * pitch / 2) + at);
#pragma unroll
      for (int q = 0; q < 4; ++q) park[k][line * LW + piece * 4 + q] = v[q];
    }
  }
  const int cl = (lane & 7) * 8, rg = wave * 8 + (lane >> 3);   // the lane's first column, and which eight rows
  const int64_t r0 = e0 + rg * 8, c0 = l0 + cl;
  uint32_t b[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) b[j] = a.scales[min(c0 + j, a.lines - 1) * (pitch / MX_BLOCK) + r0 / MX_BLOCK];
  __syncthreads();
  if (r0 >= a.length || c0 >= a.lines) return;
  typename Eight<T>::type o[8];   // by column
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    uint32_t c[BITS / 4];
#pragma unroll
    for (int k = 0; k < BITS / 4; ++k) c[k] = park[k][(cl + j) * LW + rg];
    decode8<BITS>(c, b[j], o[j]);
  }
#pragma unroll
  for (int r = 0; r < 8; ++r) {
    if (r0 + r >= a.length) break;
    typename Eight<T>::type v;
    if constexpr (sizeof(T) == 2) {
#pragma unroll
      for (int j = 0; j < 4; ++j) v[j] = __builtin_amdgcn_perm(o[2 * j + 1][r / 2], o[2 * j][r / 2], (r & 1) ? 0x07060302u : 0x05040100u);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = o[j][r];
    }
    store8(reinterpret_cast<T*>(a.x) + (r0 + r) * a.ld + c0, v, a.lines - c0);
  }
}

template <class T, int ROW, int COL>
void launch_tiles(const QuantArgs& a, hipStream_t s) {
  const int tiles_c = (int)(mx_pitch_of(a.cols) * sizeof(T) / 256);   // up to the pitches: what lies behind the ends is written too
  const int64_t tiles = tiles_c * (mx_pitch_of(a.rows) / 256);
  if (tiles >= fp4_compute_units_of_current_device())
    hipLaunchKernelGGL((mx_tile_kernel<T, ROW, COL, 8>), dim3((unsigned)((tiles + 7) / 8 * 8)), dim3(8 * 64), 0, s, a, tiles_c, tiles);
  else
    hipLaunchKernelGGL((mx_tile_kernel<T, ROW, COL, 2>), dim3((unsigned)((4 * tiles + 7) / 8 * 8)), dim3(2 * 64), 0, s, a, tiles_c, 4 * tiles);
}
template <class T, int ROW>
void launch_tiles(const QuantArgs& a, int col_bits, hipStream_t s) {
  if (col_bits == 4) launch_tiles<T, ROW, 4>(a, s);
  else launch_tiles<T, ROW, 8>(a, s);
}

template <class T>
int launch_quantize(const QuantArgs& a, int row_bits, int col_bits, hipStream_t s) {
  if (row_bits == NO_AXIS && col_bits == NO_AXIS) return FP4_OK;
  if (col_bits == NO_AXIS) {
    const int per_row = (int)(mx_pitch_of(a.cols) / MX_PITCH);
    const int64_t units = a.rows * per_row;
    const dim3 grid((unsigned)((units + 4 * ROWS_U - 1) / (4 * ROWS_U)));
    if (row_bits == 4) hipLaunchKernelGGL((mx_rows_kernel<T, 4>), grid, dim3(256), 0, s, a, units, per_row);
    else hipLaunchKernelGGL((mx_rows_kernel<T, 8>), grid, dim3(256), 0, s, a, units, per_row);
  } else if (row_bits == NO_AXIS) launch_tiles<T, NO_AXIS>(a, col_bits, s);
  else if (row_bits == 4) launch_tiles<T, 4>(a, col_bits, s);
  else launch_tiles<T, 8>(a, col_bits, s);
  FP4_CHECK_LAUNCH();
  return FP4_OK;
}

template <class T, int BITS>
int launch_dequantize(const DequantArgs& a, bool transposed, hipStream_t s) {
  if (transposed) {
    const int tiles_l = (int)((a.lines + 63) / 64);
    const int64_t tiles = tiles_l * ((a.length + 255) / 256);
    hipLaunchKernelGGL((mx_restore_cols_kernel<T, BITS>), dim3((unsigned)((tiles + 7) / 8 * 8)), dim3(256), 0, s, a, tiles_l, tiles);
  } else {
    const int per_line = (int)(mx_pitch_of(a.length) / MX_PITCH);
    const int64_t units = a.lines * per_line;
    hipLaunchKernelGGL((mx_restore_rows_kernel<T, BITS>), dim3((unsigned)((units + 4 * ROWS_U - 1) / (4 * ROWS_U))), dim3(256), 0, s, a, units, per_line);
  }
  FP4_CHECK_LAUNCH();
  return FP4_OK;
}

}  // namespace

// row_bits / col_bits: 4 or 8, or 0 where that axis is not wanted.  rows and cols are at least 1.
int mx_launch_quantize(const void* x, int bf16, int64_t rows, int64_t cols, int64_t ld, int row_bits, uint8_t* row_codes, uint8_t* row_scales,
                       int col_bits, uint8_t* col_codes, uint8_t* col_scales, hipStream_t s) {
  const QuantArgs a = {x, rows, cols, ld, row_codes, row_scales, col_codes, col_scales};
  return bf16 ? launch_quantize<uint16_t>(a, row_bits, col_bits, s) : launch_quantize<float>(a, row_bits, col_bits, s);
}

int mx_launch_dequantize(const uint8_t* codes, const uint8_t* scales, int bits, int64_t lines, int64_t length, bool transposed, void* x, int bf16,
                         int64_t ld, hipStream_t s) {
  const DequantArgs a = {codes, scales, x, lines, length, ld};
  if (bf16) return bits == 4 ? launch_dequantize<uint16_t, 4>(a, transposed, s) : launch_dequantize<uint16_t, 8>(a, transposed, s);
  return bits == 4 ? launch_dequantize<float, 4>(a, transposed, s) : launch_dequantize<float, 8>(a, transposed, s);
}
