// Which kernel takes an MX product: host arithmetic on its sizes and the number of compute units.
#pragma once
#include <stdint.h>

#include <algorithm>

struct MxTiling {
  int tile;   // 16: few tokens (mx_few.hip); 32: tiles whose waves share the contraction; 64, 128, 256: rows and columns of a tile
  int rest;   // 256: tiles of the last round that are cut into 128 x 128 ones
};

inline MxTiling mx_gemm_tiling(int64_t P, int64_t Q, int64_t Kc, int bits_l, int bits_r, int n_cu) {
  if (Kc == 0) return {64, 0};
  const int64_t passes = (bits_l / 4) * (bits_r / 4);
  if (P <= 32 || (P <= 64 && Kc * passes <= 2048)) return {16, 0};
  const int64_t t32 = ((P + 31) / 32) * ((Q + 31) / 32), t128 = ((P + 127) / 128) * ((Q + 127) / 128), t256 = ((P + 255) / 256) * ((Q + 255) / 256);
  const int64_t t64 = ((P + 63) / 64) * ((Q + 63) / 64), steps = (Kc + 511) / 512 * 2 * passes;   // of 256 codes
  if (t32 > 2 * (int64_t)n_cu && t64 <= n_cu && steps <= 4) return {64, 0};
  if (t32 <= 4 * (int64_t)n_cu) return {32, 0};
  if (t128 <= n_cu) return {128, 0};
  const int64_t wgs = n_cu / 8 * 8;
  return {256, (int)(t256 > wgs && 4 * (t256 % wgs) <= wgs ? t256 % wgs : 0)};
}
