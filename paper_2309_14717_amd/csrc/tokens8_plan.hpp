// Launch shape of the kernel that brings rows to 8 bits (tokens8.hip).
#pragma once
#include <stddef.h>

namespace qalora {

constexpr int T8_MAX_COLS = 1 << 17;  // 1024 threads with sixteen pieces of eight columns each
constexpr int T8_MOST_ROWS = 1 << 21;  // of a launch

struct Tokens8Plan {
  int lanes;   // threads along a row: 64, 256 or 1024
  int pieces;  // of eight columns, a thread's at most: 1, 2, 4, 8 or 16
  int rows;    // of a block
};
inline Tokens8Plan tokens8_plan(int cols) {
  const int eights = (cols + 7) / 8;
  Tokens8Plan p{};
  p.lanes = eights <= 128 ? 64 : (eights <= 1024 ? 256 : 1024);
  p.pieces = 1;
  while (p.pieces * p.lanes < eights) p.pieces *= 2;
  p.rows = p.lanes == 64 ? 4 : 1;
  return p;
}

}  // namespace qalora
