// Which products of few tokens stream the weight, and bring the tokens to 8 bits in the same launch (stream_i8.hip).
#pragma once
#include <stddef.h>

namespace qalora {

constexpr int S8_COLS = 16;  // of a block
constexpr int S8_WAVES = 8;  // each with every eighth 128 bytes of the rows
constexpr int S8_TOKENS = 16;
constexpr int S8_ELEMENTS = 16384;  // of all tokens: every block brings them to 8 bits, at LDS bytes as many
constexpr int S8_AT_ONCE = 3;       // blocks of a compute unit

// One launch saves one, and every block makes the codes again, of which the other blocks of its unit hide the less the more there are.
// One launch and two, us, the weight from memory: 16 tokens of 1024 to 1024, 4096, 8192 and 22016 channels 6.2 / 6.9, 6.8 / 7.1, 8.8 / 7.3,
// 19.4 / 10.0; 8 tokens to 8192 and 9216 6.5 / 7.3, 8.2 / 7.4; 4 tokens of 4096 to 8192 and 9216 12.1 / 12.9, 15.8 / 14.0; 2 tokens
// of 8192 to 12288 and 16384 21.4 / 24.1, 29.0 / 30.1 (28672: 46.1 / 44.9).  Where a unit has more blocks than it holds, one token alone, of
// rows long enough for the weight to take the time: 1024 to 16384 8.8 / 7.6, to 65536 23.4 / 15.5, 4096 to 22016 20.1 / 23.7, to
// 65536 51.5 / 54.9, 8192 to 22016 34.3 / 36.3.
inline bool stream8_takes(int tokens, int K, int N) {
  const size_t elements = (size_t)tokens * K;
  if (tokens > S8_TOKENS || elements > S8_ELEMENTS) return false;
  const int blocks = (N + S8_COLS * 256 - 1) / (S8_COLS * 256);  // a unit's
  if (blocks > S8_AT_ONCE) return tokens == 1 && K >= 4096;
  return elements * blocks <= S8_ELEMENTS || tokens * blocks <= 8;
}

}  // namespace qalora
