// Launch shape and workspace of the orthogonalised update (muon.hip).
#pragma once
#include <stddef.h>
#include <stdint.h>

namespace qalora {

constexpr int MUON_MAX_TENSORS = 32;
constexpr int MUON_MAX_SHORT = 128;  // shorter side of a matrix: its Gram matrix lives in one compute unit's LDS
constexpr int MUON_CHUNK = 64;       // entries of the longer side that a block works on at a time

// One matrix, seen as X [shorter side x longer side].
struct MuonTensor {
  float *p, *g, *m;      // [rows, cols]
  int rows, cols;
  int tiles;             // 32-row tiles of the shorter side
  int chunks;            // of the longer side
  float step_size;       // lr times the shape's scale
  size_t x;              // floats from the workspace's start: X as [chunks][32 tiles][MUON_CHUNK]
  size_t gram;           // the Gram matrix: [tiles][tiles] of 32 x 32
  size_t partial;        // each block's share of it
};
struct MuonTable {
  int n, blocks, reduce_blocks, per_block, max_tiles;
  int block0[MUON_MAX_TENSORS];   // first block of the launches over X; blocks of `per_block` chunks
  int reduce0[MUON_MAX_TENSORS];  // first block of the launch that adds the blocks' Gram matrices
  MuonTensor t[MUON_MAX_TENSORS];
};
constexpr int MUON_REDUCE_BLOCKS_PER_TILE = 8;  // (muon_reduce_kernel: 32 of a tile's 256 16-byte pieces a block)

// Blocks over X: about as many as the chip holds at once (a block first squares the Gram matrix, so more of them only
// repeat that; 143 KB of LDS with more than 64 rows, 55 KB below).
constexpr int muon_target_blocks(int max_tiles) { return max_tiles > 2 ? 256 : 512; }

// Fills in the table from rows[] and cols[]; returns the workspace's floats, 0 where the list is not acceptable
// (`unsupported` says whether a matrix has both sides above MUON_MAX_SHORT, rather than a bad argument).
inline size_t muon_table(int n, const int32_t* rows, const int32_t* cols, MuonTable& table, bool& unsupported) {
  unsupported = false;
  if (n < 1 || n > MUON_MAX_TENSORS || !rows || !cols) return 0;
  long long chunks = 0;
  table.n = n;
  table.max_tiles = 0;
  for (int i = 0; i < n; ++i) {
    if (rows[i] < 1 || cols[i] < 1) return 0;
    MuonTensor& t = table.t[i];
    t.rows = rows[i];
    t.cols = cols[i];
    const int shorter = rows[i] < cols[i] ? rows[i] : cols[i], longer = rows[i] < cols[i] ? cols[i] : rows[i];
    if (shorter > MUON_MAX_SHORT) unsupported = true;
    t.tiles = (shorter + 31) / 32;
    t.chunks = longer / MUON_CHUNK + (longer % MUON_CHUNK ? 1 : 0);
    if (t.tiles > table.max_tiles) table.max_tiles = t.tiles;
    chunks += t.chunks;
  }
  if (unsupported) return 0;
  const int target = muon_target_blocks(table.max_tiles);
  table.per_block = (int)((chunks + target - 1) / target);
  size_t floats = 0;
  table.blocks = table.reduce_blocks = 0;
  for (int i = 0; i < n; ++i) {
    MuonTensor& t = table.t[i];
    const int blocks = (t.chunks + table.per_block - 1) / table.per_block;
    const size_t gram = (size_t)t.tiles * t.tiles * 1024;
    table.block0[i] = table.blocks;
    table.reduce0[i] = table.reduce_blocks;
    table.blocks += blocks;
    table.reduce_blocks += t.tiles * t.tiles * MUON_REDUCE_BLOCKS_PER_TILE;
    t.x = floats;
    floats += (size_t)t.chunks * t.tiles * 32 * MUON_CHUNK;
    t.gram = floats;
    floats += gram;
    t.partial = floats;
    floats += (size_t)blocks * gram;
  }
  for (int i = n; i < MUON_MAX_TENSORS; ++i) table.block0[i] = table.reduce0[i] = INT32_MAX;
  return floats;
}

}  // namespace qalora
