// Launch shape of the kernel that brings rows to 8 bits (tokens8.hip).
#pragma once
#include <stddef.h>

namespace qalora {

constexpr int T8_MAX_COLS = 1 << 17;  // 1024 threads with sixteen pieces of eight columns each
constexpr int T8_MOST_ROWS = 1 << 21;  // of a launch

struct Tokens8Plan {
  int lanes;   // threads along a row: 64, 256, 512 or 1024
  int pieces;  // of eight columns, a thread's at most
  int rows;    // of a block at once
};
// Many rows: as few threads a row as hold it in four pieces each, so that a compute unit has many rows on their way (4096 rows of 11008 with
// factors: 26.6 us with 512 threads of three pieces, 30.6 with 256 of six, 35.3 with 1024 of two); few rows: as many threads as there are.
constexpr int T8_MANY_ROWS = 512;
inline Tokens8Plan tokens8_plan(int rows, int cols) {
  const int eights = (cols + 7) / 8;
  Tokens8Plan p{};
  const bool many = rows > T8_MANY_ROWS;
  p.lanes = eights <= (many ? 128 : 64) ? 64 : eights <= (many ? 512 : 256) ? 256 : many && eights <= 2048 ? 512 : 1024;
  const int need = (eights + p.lanes - 1) / p.lanes;
  p.pieces = need <= 2 || (need == 3 && p.lanes == 512) ? need : need <= 4 ? 4 : need <= 8 ? 8 : 16;
  p.rows = p.lanes == 64 ? 4 : 1;
  return p;
}
// Blocks of a launch at most: where a row's loads wait for more than its bytes (factors, hidden activations), as many as the chip has room for
// at once, each with every so manyth row, the next on its way meanwhile (4096 rows of 11008 with factors: 768 blocks 26.6 us, a block
// a row 31.1; of 13824 512 blocks 34.9, 768 42.2; 1531 of 22016 hidden activations: 256 blocks 36.1, 512 41.3).  Plain rows: a block
// for each (4096 of 4096: 12.5 us, and 14.6 with 1024 blocks).
inline int tokens8_blocks(const Tokens8Plan& p, int rows, bool plain, bool swiglu) {
  if (plain || rows <= T8_MANY_ROWS) return T8_MOST_ROWS;
  if (p.lanes <= 256) return (swiglu ? 512 : 768) * 4;
  if (p.lanes == 512) return p.pieces == 2 ? 1024 : p.pieces == 3 && !swiglu ? 768 : 512;
  return swiglu ? 256 : 512;
}

}  // namespace qalora
