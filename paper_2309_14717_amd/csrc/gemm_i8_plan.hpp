// Which tile a product of 8-bit integers takes, and into how many slices its K is split (gemm_i8.hip).
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>

namespace qalora {

constexpr int I8_STEP = 128;    // of K
constexpr int I8_MAX_SLICES = 32;
constexpr size_t I8_MAX_PARTIALS = (size_t)32 << 20;  // bytes of the slices' sums
constexpr int I8_MAX_TOKENS = 1 << 29;

enum { I8_256x256, I8_192x256, I8_128x256, I8_128x128, I8_128x64, I8_64x128, I8_64x64, I8_32x128, I8_32x64, I8_16x128, I8_16x64, I8_TILES };
// Tokens by columns; threads; blocks of a compute unit at once (LDS); and what a step of 128 takes, in ns, forward and backward, of a
// block that has its unit to itself, and per block where there are as many as fit (0: not in this direction).  Measured with weights
// that no cache holds, at sizes from 16 x 4096 x 4096 to 4096 x 11008 x 4096.  Up to 32 tokens the backward takes 128 columns, so that it
// reads whole cache lines of a weight's rows (16 x 11008 x 4096: 14.1 us, with 64 columns 21), the forward 64 for more blocks.
struct Int8Tile {
  int rows, cols, threads, at_once;
  int alone[2], shared[2];
};
constexpr Int8Tile kInt8Tiles[I8_TILES] = {
    {256, 256, 512, 1, {1670, 1670}, {1670, 1670}},
    {192, 256, 512, 1, {1400, 1400}, {1400, 1400}},
    {128, 256, 512, 1, {950, 1000}, {950, 1000}},
    {128, 128, 512, 2, {700, 720}, {500, 520}},
    {128, 64, 512, 2, {470, 0}, {400, 0}},
    {64, 128, 256, 2, {490, 600}, {420, 600}},
    {64, 64, 256, 2, {400, 0}, {330, 0}},
    {32, 128, 256, 2, {0, 520}, {0, 560}},
    {32, 64, 128, 3, {330, 0}, {270, 0}},
    {16, 128, 128, 2, {0, 500}, {0, 540}},
    {16, 64, 128, 4, {285, 0}, {250, 0}},
};

struct Int8Plan {
  int tile, slices;
};
inline Int8Plan int8_plan(int M, int N, int K, bool back) {
  const long steps = (K + I8_STEP - 1) / I8_STEP;
  Int8Plan best{I8_256x256, 1};
  double least = 1e30;
  for (int t = I8_TILES - 1; t >= 0; --t) {  // (the smaller one of two that are as fast)
    const Int8Tile& tile = kInt8Tiles[t];
    if (tile.alone[back] == 0 || (tile.rows > 16 && tile.rows >= 2l * M)) continue;  // (rows that are not there cost LDS and its traffic)
    const long tiles = (((long)M + tile.rows - 1) / tile.rows) * ((N + tile.cols - 1) / tile.cols);
    if (t != I8_256x256 && tiles * tile.threads >= 1l << 31) continue;  // (a launch has at most 2^32 threads)
    for (int s = 1; s <= I8_MAX_SLICES && s <= steps; ++s) {
      if (s > 1 && ((size_t)s * M * N * 4 > I8_MAX_PARTIALS || tiles * s > 1024)) break;
      const long per = (steps + s - 1) / s;
      if ((steps + per - 1) / per != s) continue;  // a slice would be empty
      const long n = (tiles * s + 255) / 256, rounds = (n + tile.at_once - 1) / tile.at_once;  // of a compute unit
      double ns = per * (double)(n * tile.shared[back] > rounds * tile.alone[back] ? n * tile.shared[back] : rounds * tile.alone[back]);
      ns += 3000.0 * rounds;  // first loads and last stores
      const double weights = (double)N * K / 4800.0;  // no faster than the weight is read
      ns = (ns < weights ? weights : ns) + 0.1 * ns;  // (of those that reach that, the one with the least to do)
      // the sum over the slices: a launch, and four bytes written and read for each element of each
      if (s > 1) ns += 4500.0 + 8.0 * s * M * N / 4000.0;
      if (ns < least) {
        least = ns;
        best = Int8Plan{t, s};
      }
    }
  }
  return best;
}
// A product of some rounds of 256 x 256 tiles and part of another: the columns of whole rounds keep them, and the others' tiles are as narrow
// as leaves them one round.  narrow = 0: all tiles alike.
struct Int8Mixed {
  int narrow, wide_n;
};
__host__ __device__ inline int int8_narrow_first(int narrow) { return narrow / 2 / 8 * 8; }
inline Int8Mixed int8_mixed(int M, int N, int slices, bool back) {
  const long tiles_m = ((long)M + 255) / 256, tiles = tiles_m * ((N + 255) / 256), rounds = tiles / 256;
  if (slices > 1 || rounds < 1 || tiles % 256 == 0 || tiles_m > 256) return Int8Mixed{0, 0};
  const int wide_n = (int)(rounds * 256 / tiles_m), rest = N - wide_n * 256;
  for (const int w : {128, 192})
    if (!(back && w == 192) && tiles_m * ((rest + w - 1) / w) <= 256) return Int8Mixed{w, wide_n};
  return Int8Mixed{0, 0};
}
// Room for the slices' sums of any number of tokens up to M.
inline size_t int8_partials(int M, int N) {
  const size_t all = (size_t)I8_MAX_SLICES * M * N * 4;
  return all < I8_MAX_PARTIALS ? all : I8_MAX_PARTIALS;
}

}  // namespace qalora
