// Which kernel takes an MX product: host arithmetic on its sizes and the number of compute units.
#pragma once
#include <stdint.h>

#include <algorithm>

struct MxTiling {
  int tile;   // 16: few tokens (mx_few.hip); 32: tiles whose waves share the contraction; 64, 128, 256: rows and columns of a tile; 192: 256 rows
  int rest;   // 256: tiles of the last round that are cut into 128 x 128 ones
};

// All lines below were drawn from some 900 products of 33 .. 8192 x 256 .. 12288 over 256 .. 13824, in 4 and 8 bits, timed by every kernel; on 422
// others the one taken is within 5 % of the best in all but 8, within 15 % in all but one.
inline MxTiling mx_gemm_tiling(int64_t P, int64_t Q, int64_t Kc, int bits_l, int bits_r, int n_cu) {
  if (Kc == 0) return {64, 0};   // nothing to request ahead: the operands may be null
  const int64_t passes = (bits_l / 4) * (bits_r / 4);
  const auto tiles = [&](int64_t rows, int64_t cols) { return ((P + rows - 1) / rows) * ((Q + cols - 1) / cols); };
  const auto rounds = [&](int64_t n) { return (n + n_cu - 1) / n_cu; };
  // Few tokens: the kernel that reads each weight once.  From 33 on the smallest tiles, which stage the tokens in LDS, catch up as the
  // contraction grows, us as few / 32: 61 x 592 over 3008 in 8 x 8 bits 14.8 / 10.0, 62 x 2488 over 10296 16.0 / 10.4, 64 x 2048 over 2048 5.8 / 5.7, 36 x
  // 4768 over 696 5.1 / 5.6, 53 x 3344 over 392 4.5 / 5.2, and with many columns: 46 x 10496 over 1960 10.1 / 8.7; up to 32 tokens they do not: 32 x
  // 5120 over 13824 19.2 / 22.
  // Where the outputs are so small that both take one round of short chains, it is ahead up to 256 tokens (163 x 448 over 408 4.2 / 4.9, 174 x 440
  // over 1008 4.6 / 5.1; with nine steps 220 x 1008 over 2080 6.2 / 5.9).
  const int64_t steps = (Kc + 255) / 256 * passes, t32 = tiles(32, 32);
  if (P <= 32 || (P <= 64 && Kc * passes <= 2048 && t32 <= 2 * (int64_t)n_cu) || (P <= 256 && t32 <= n_cu && steps <= 4)) return {16, 0};
  // One or two workgroups' worth of steps: operands straight from memory (1332 x 680 over 432: 64 / 32 tiles 5.7 / 8.1 us, 2114 x 432 over 736
  // 6.9 / 8.7; where the 32 x 32 ones go round the chip twice at most they are as fast: 512 x 512 over 512 5.3 / 5.1).
  if (t32 > 2 * (int64_t)n_cu && tiles(64, 64) <= n_cu && steps <= 4) return {64, 0};
  // Small outputs are one chain of round trips a tile: four times the workgroups, whose waves share it, win up to four of them a CU (32 / 128
  // tiles: 69 x 6808 over 5384 13.3 / 20 us, 857 x 592 over 9304 19.8 / 31, 1024 x 1024 over 4096 15.4 / 16.1; past it 164 x 5496 over 1832 12.0 / 11.4, 861 x
  // 1720 over 10792 47 / 36).
  if (t32 <= 4 * (int64_t)n_cu) return {32, 0};
  // The larger tiles, in hundredths of a us (measured): 128 x 128 rounds of them, each a start and end and so much a step; the others, whose
  // workgroups go on to their next tile while they store one, a start and end once and less a round, and more a step the more of the
  // CUs draw on memory (256 columns: 1.3 us with 8 tiles, 1.37 with 120, 1.43 with 176 of 256, 1.62 with 210, 1.85 with 256; 192: 1.1 with 8, 1.2
  // with 180, 1.34 with 232, 1.4 with 256).  Their steps come in pairs.
  const int64_t pairs = (Kc + 511) / 512 * 2 * passes, wgs = n_cu / 8 * 8, t256 = tiles(256, 256);
  const auto many = [&](int64_t n, int64_t least, int64_t most, int64_t from) {   // n tiles; from: the share of the CUs, in per cent, to which a step takes the least
    const int64_t share = 100 * (n % wgs) / wgs, step = least + std::max<int64_t>(share - from, 0) * (most - least) / (100 - from);
    return n / wgs * (450 + most * pairs) + (n % wgs ? 450 + step * pairs : 0);
  };
  const int64_t cost128 = rounds(tiles(128, 128)) * (500 + 68 * steps), cost192 = 510 + many(tiles(256, 192), 110, 140, 40);
  // A last round of 256 x 256 tiles that a quarter of the CUs have at most is cut into 128 x 128 ones, in a launch of its own.
  const int64_t rest = t256 > wgs && 4 * (t256 % wgs) <= wgs ? t256 % wgs : 0;
  const int64_t cost256 = 510 + many(t256 - rest, 130, 185, 60) + (rest ? 700 + 68 * steps : 0);
  if (cost128 <= std::min(cost192, cost256)) return {128, 0};
  return cost192 < cost256 ? MxTiling{192, 0} : MxTiling{256, (int)rest};
}
