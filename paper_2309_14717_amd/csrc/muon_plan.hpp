// Launch shape and workspace of the orthogonalised update (muon.hip).
#pragma once
#include <stddef.h>
#include <stdint.h>

namespace qalora {

constexpr int MUON_MAX_TENSORS = 32;
constexpr int MUON_MAX_SHORT = 128;  // shorter side of a matrix: its Gram matrix lives in one compute unit's LDS
constexpr int MUON_MAX_LONG = 1 << 27;  // a lane's distance in bytes from its wavefront's first element fits 32 bits
constexpr int MUON_CHUNK = 32;       // entries of the longer side that a wavefront works on at a time

// One matrix, seen as X [shorter side x longer side].
struct MuonTensor {
  float *p, *g, *m;      // [rows, cols]
  int rows, cols;
  int chunks;            // of the longer side
  float step_size;       // lr times the shape's scale
  size_t x;              // floats from the workspace's start: X as [chunks][tiles] of 32 x MUON_CHUNK
  size_t gram;           // the Gram matrix: [tiles][tiles] of 32 x 32
  size_t partial;        // each block's share of it: the upper tiles (in two places where `direct`)
};
struct MuonTable {
  int n, blocks, reduce_blocks, per_block;
  int tiles;                      // 32-row tiles that every X has: 1, 2 or 4, rows beyond a shorter side being zero
  bool alone;                     // a block does all steps of a matrix
  bool direct;                    // blocks add their matrix's shares of G by themselves
  int block0[MUON_MAX_TENSORS];   // first block of the launches over X; blocks of `per_block` chunks
  int reduce0[MUON_MAX_TENSORS];  // first block of the launch that adds the blocks' Gram matrices
  MuonTensor t[MUON_MAX_TENSORS];
};
constexpr int MUON_REDUCE_BLOCKS_PER_TILE = 8;  // (muon_reduce_kernel: 32 of a tile's 256 16-byte pieces a block)
constexpr int muon_upper_tiles(int tiles) { return tiles * (tiles + 1) / 2; }

// A block's wavefronts take `muon_waves` chunks at a time; blocks over X as many as there are compute units at most (a block first
// makes P from the Gram matrix, and leaves a share of the next: more of them only repeat that).
constexpr int muon_waves_of(int tiles) { return tiles > 2 ? 4 : 8; }
constexpr int MUON_BLOCKS = 256;
// One launch, a block for each matrix, where the longest has this many 32 x 32 tiles of X at most; and no launches that add the
// blocks' shares of G, but every block for itself, where that is this many tiles at most.  Two matrices, 5 steps, us, with one launch, six
// and eleven: 32 x 512 25 / 30 / 42, 768 32 / 32 / 42, 1024 38 / 34 / 42, 4096 - / 34 / 45, 11008 - / 46 / 53, 16384 - / 51 / 49;
// 64 x 384 39 / 46 / 56, 640 53 / 50 / 56, 4096 - / 59 / 60, 8192 - / 75 / 65.  Fourteen likewise.
// Neither beyond 64 rows: G and P take 64 KB each there, and with the 68 KB that the last pass keeps for tall matrices, or the 80 KB of a
// block's shares, more than the 160 KB of a compute unit (so two of 65 x 1024 take 99 us where two of 64 x 1024 take 53).
// Both hold for the list, by its longest matrix, as do the tiles by its largest shorter side: a launch is one kernel for all matrices, and one
// that a single matrix needs is made anyhow.  13 of 32 x 4096 and one of 32 x 22016: 58 in one list, 42 + 50 in two; 13 of 64 x 1024 and
// one of 64 x 11008 72, 57 + 66.  Padding to the largest shorter side can cost that much: 14 of rank 16 and one of 128 x 4096 take 168, 48 + 103
// in two lists.
constexpr int MUON_ALONE_TILES = 24;
constexpr int MUON_DIRECT_TILES = 48;

// Fills in the table from rows[] and cols[]; returns the workspace's floats, 0 where the list is not acceptable
// (`unsupported` says whether a matrix has both sides above MUON_MAX_SHORT, rather than a bad argument).
inline size_t muon_table(int n, const int32_t* rows, const int32_t* cols, MuonTable& table, bool& unsupported) {
  unsupported = false;
  if (n < 1 || n > MUON_MAX_TENSORS || !rows || !cols) return 0;
  long long chunks = 0;
  table.n = n;
  int longest = 0, most_chunks = 0;
  for (int i = 0; i < n; ++i) {
    if (rows[i] < 1 || cols[i] < 1) return 0;
    if (rows[i] > MUON_MAX_LONG || cols[i] > MUON_MAX_LONG) unsupported = true;
    MuonTensor& t = table.t[i];
    t.rows = rows[i];
    t.cols = cols[i];
    const int shorter = rows[i] < cols[i] ? rows[i] : cols[i], longer = rows[i] < cols[i] ? cols[i] : rows[i];
    if (shorter > MUON_MAX_SHORT) unsupported = true;
    if (shorter > longest) longest = shorter;
    t.chunks = longer / MUON_CHUNK + (longer % MUON_CHUNK ? 1 : 0);
    chunks += t.chunks;
    if (t.chunks > most_chunks) most_chunks = t.chunks;
  }
  if (unsupported) return 0;
  table.tiles = longest > 64 ? 4 : (longest > 32 ? 2 : 1);
  table.alone = table.tiles <= 2 && most_chunks <= MUON_ALONE_TILES / table.tiles;
  const int waves = muon_waves_of(table.tiles), upper = muon_upper_tiles(table.tiles);
  table.per_block = (int)((chunks + MUON_BLOCKS * waves - 1) / (MUON_BLOCKS * waves)) * waves;
  table.direct = table.tiles <= 2 && (most_chunks + table.per_block - 1) / table.per_block * upper <= MUON_DIRECT_TILES;
  size_t floats = 0;
  table.blocks = table.reduce_blocks = 0;
  for (int i = 0; i < n; ++i) {
    MuonTensor& t = table.t[i];
    const int blocks = (t.chunks + table.per_block - 1) / table.per_block;
    table.block0[i] = table.blocks;
    table.reduce0[i] = table.reduce_blocks;
    table.blocks += blocks;
    table.reduce_blocks += upper * MUON_REDUCE_BLOCKS_PER_TILE;
    t.x = floats;
    floats += (size_t)t.chunks * table.tiles * 32 * MUON_CHUNK;
    t.gram = floats;
    floats += (size_t)table.tiles * table.tiles * 1024;
    t.partial = floats;
    floats += (size_t)blocks * upper * 1024 * (table.direct ? 2 : 1);
  }
  for (int i = n; i < MUON_MAX_TENSORS; ++i) table.block0[i] = table.reduce0[i] = INT32_MAX;
  return floats;
}

}  // namespace qalora
