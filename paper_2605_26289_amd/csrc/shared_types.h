// Descriptors of attention for batches that share cells (device memory layout, plain structs).  Positions are logical token
// positions inside a sequence.
#pragma once
#include <stdint.h>

namespace dk {
constexpr int32_t SHARED_BLOB_BYTES = 3584;  // descriptors up to this size travel in a kernel's arguments
}  // namespace dk

// Rows against a range of positions that all of them see through the same cells: a prefix that several entries share, or what
// one entry has to itself, its new tokens included.  Its work items are pieces of `chunk` keys times row tiles, the tiles of a piece
// side by side; piece s of row r leaves its sums in partial row part0 + s * rows + r.
struct DkShNode {
  int32_t tok0;   // of one entry: its first packed token; shared: place of the first token in the table of tokens
  int32_t rows;   // packed rows: tokens x query heads of a KV head
  int32_t lo, keys;
  int32_t chunk;  // a multiple of 64
  int32_t seg0;   // its segments: up to the next node's first
  int32_t part0;  // -1: the rows are complete, to be stored as output
  int32_t n;      // of one entry: the position of its first new token; shared: SHARED_ALL, every row sees every key
};

// A run of cells with positions pos .. pos + len - 1.  start < 0: staged new tokens, from row ~start on.
struct DkShSeg {
  int32_t start, pos, len;
};

// One of the prefixes in front of an entry's own range, for the merge of its rows.
struct DkShSource {
  int32_t part0;  // of the entry's first row, in the first piece
  int32_t step;   // partial rows from piece to piece
  int32_t pieces;
};

namespace dk {
constexpr int32_t SHARED_ALL = 1 << 30;  // DkShNode::n of a shared range
constexpr int32_t SHARED_TILE = 128;     // rows of a tile of the bf16 kernel; nodes of up to SHARED_FEW rows are one tile
constexpr int32_t SHARED_FEW = 64;
}  // namespace dk
