// Which products of few tokens stream the weight, and bring the tokens to 8 bits in the same launch (stream_i8.hip).
#pragma once
#include <stddef.h>

namespace qalora {

constexpr int S8_COLS = 16;  // of a block
constexpr int S8_WAVES = 8;  // each with every eighth 128 bytes of the rows
constexpr int S8_TOKENS = 16;
constexpr int S8_ELEMENTS = 16384;  // of all tokens: every block brings them to 8 bits, at LDS bytes as many

// One launch saves one, and every block makes the codes again, of which the other blocks of its unit hide the less the more there are.
// Calls one after the other from the host, of which one with two launches takes 9 to 10 us whatever it does, and one with one 6; in
// brackets the same in a graph.  One launch and two, us, the weight from memory:
//   two blocks a unit    16 tokens, 1024 -> 8192 9.0 / 10.5 (8.9 / 7.3);  4, 4096 -> 8192 12.2 / 15.0 (12.3 / 12.6)
//   three, all at once   8, 1024 -> 12288 8.3 / 10.2 (8.1 / 7.6);  16 11.3 / 9.8 (11.2 / 7.7);  2, 8192 -> 12288 21.2 / 23.3 (20.9 / 23.0);
//                        4, 4096 -> 12288 15.9 / 15.3 (16.0 / 14.6)
//   four to six          4, 1024 -> 13824 8.8 / 9.6 (8.7 / 7.8);  16 14.2 / 10.0 (14.2 / 7.7);  16, 1024 -> 22016 17.6 / 10.7 (17.8 / 9.8);
//                        2, 2560 -> 13824 13.7 / 11.7 (13.6 / 11.1);  one token, 8192 -> 22016 33.2 / 35.0 (33.0 / 34.7)
//   more                 1, 1024 -> 65536 23.1 / 16.5 (23.5 / 15.2);  16 47.1 / 16.1 (47.0 / 15.6);  1, 4096 -> 65536 49.9 / 52.8 (49.8 / 52.5)
inline bool stream8_takes(int tokens, int K, int N) {
  const size_t elements = (size_t)tokens * K;
  if (tokens > S8_TOKENS || elements > S8_ELEMENTS) return false;
  const int blocks = (N + S8_COLS * 256 - 1) / (S8_COLS * 256);  // a unit's
  if (blocks <= 2) return true;
  if (blocks == 3) return tokens <= 2 || elements <= 8192;
  if (tokens == 1 && K >= 4096) return true;  // (the weight's bytes take the time)
  return blocks <= 6 && K <= 1024 && elements * blocks <= 16384;
}

}  // namespace qalora
