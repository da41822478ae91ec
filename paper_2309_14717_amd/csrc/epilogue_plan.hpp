// Launch shape and workspace of the epilogue's backward (epilogue.hip).
#pragma once
#include <stddef.h>

namespace qalora {

constexpr int EB_THREADS = 256;
constexpr int EB_MAX_LANES = 64;  // of eight columns each: a row of a block's tile is up to 1 KB of bf16
constexpr int EB_MIN_LANES = 8;   // 128 bytes
constexpr int EB_ONE_BLOCK_ROWS = 256;
constexpr int EB_MAX_COLS = 1 << 29;  // a launch has at most 2^32 threads, and narrow tiles take four to a column

struct EpilogueBackPlan {
  int lanes;       // threads along a row (a power of two); the block takes EB_THREADS / lanes rows at a time
  int col_blocks;
  int row_blocks;  // each of `rows_per` rows
  int rows_per;
};
inline EpilogueBackPlan epilogue_back_plan(int rows, int cols) {
  EpilogueBackPlan p{};
  const int eights = cols / 8;
  // Few rows: narrow tiles, so that one block has all rows of its columns and dbias needs no second launch
  p.lanes = rows <= EB_ONE_BLOCK_ROWS ? EB_MIN_LANES : EB_MAX_LANES;
  while (p.lanes > EB_MIN_LANES && p.lanes / 2 >= eights) p.lanes /= 2;
  p.col_blocks = (eights + p.lanes - 1) / p.lanes;
  const int at_once = EB_THREADS / p.lanes;
  const int want = (2048 + p.col_blocks - 1) / p.col_blocks;  // eight blocks per compute unit
  const int sweeps = rows / at_once + (rows % at_once ? 1 : 0);
  const int sweeps_per = rows <= EB_ONE_BLOCK_ROWS ? sweeps : (sweeps / want > 4 ? sweeps / want + 1 : 4);
  p.rows_per = sweeps_per * at_once;
  p.row_blocks = sweeps / sweeps_per + (sweeps % sweeps_per ? 1 : 0);
  return p;
}
// The row blocks' shares of dbias (none where there is one).
inline size_t epilogue_back_floats(int rows, int cols) {
  const size_t blocks = epilogue_back_plan(rows, cols).row_blocks;
  return blocks > 1 ? blocks * cols : 0;
}

}  // namespace qalora
