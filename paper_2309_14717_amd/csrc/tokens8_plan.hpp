// Launch shape of the kernel that brings rows to 8 bits (tokens8.hip).
#pragma once
#include <stddef.h>

namespace qalora {

constexpr int T8_MAX_COLS = 1 << 17;  // 1024 threads with sixteen pieces of eight columns each
constexpr int T8_MOST_ROWS = 1 << 21;  // of a launch

struct Tokens8Plan {
  int lanes;   // threads along a row: 64, 256 or 1024
  int pieces;  // of eight columns, a thread's at most
  int rows;    // of a block
};
// Many rows: as few threads a row as hold it, so that a compute unit has many rows on their way; few rows: as many threads as there are.
inline Tokens8Plan tokens8_plan(int rows, int cols) {
  const int eights = (cols + 7) / 8;
  Tokens8Plan p{};
  const bool many = rows > 512;
  p.lanes = eights <= (many ? 128 : 64) ? 64 : (eights <= (many ? 256 * 12 : 256) ? 256 : 1024);
  const int need = (eights + p.lanes - 1) / p.lanes;
  constexpr int kHeld[] = {1, 2, 3, 4, 6, 8, 12, 16};
  for (const int h : kHeld)
    if (h >= need && !(p.lanes == 1024 && (h == 3 || h == 6 || h == 12))) {
      p.pieces = h;
      break;
    }
  p.rows = p.lanes == 64 ? 4 : 1;
  return p;
}

}  // namespace qalora
