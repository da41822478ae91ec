// Which products of few tokens stream the weight, and bring the tokens to 8 bits in the same launch (stream_i8.hip).
#pragma once
#include <stddef.h>

namespace qalora {

constexpr int S8_COLS = 16;  // of a block
constexpr int S8_WAVES = 8;  // each with every eighth 128 bytes of the rows
constexpr int S8_TOKENS = 16;
constexpr int S8_ELEMENTS = 16384;  // of all tokens: every block brings them to 8 bits, at LDS bytes as many

inline bool stream8_takes(int tokens, int K) { return tokens <= S8_TOKENS && (size_t)tokens * K <= S8_ELEMENTS; }

}  // namespace qalora
