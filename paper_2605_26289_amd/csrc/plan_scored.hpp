// Host-side planning of one dk_scored_attend call: slots to segments, what every row sees, the descriptors' layout.
#pragma once
#include <cstddef>
#include <cstdint>
#include <vector>

#include "device_types.h"
#include "pool.hpp"

namespace dk {

// Which positions the rows of a call see, besides causality (HOST arrays, null: no such mask).
struct ScoreMasks {
  int32_t window = 0;               // > 0: a row sees its own position and window - 1 before it
  const int64_t* prefix = nullptr;  // [n_seqs]: every row of the entry sees positions below it
  const int64_t* first = nullptr;   // [tokens]: the row sees no position below it
};

// What the cuts go by.
struct ScoredConfig {
  int32_t n_q_heads = 0, n_kv_heads = 0, head_dim = 0;
  bool bf16 = true;
  int32_t few_rows = 64;     // bf16: entries of at most this many packed rows go to the kernel for few rows
  // Smallest key range worth a work item there, and in the rows kernels.  Measured, us, 128 / 256 / 512: one bf16 token on 600 9.0 / 9.9 /
  // 10.8, on 3000 13.5 / 10.8 / 12.4, on 10 000 19.6 / 19.5 / 17.8, of 64-wide heads on 3000 12.1 / 9.4 / 10.2; one fp32 token on 5000
  // 18.1 / 17.7 / 22.1, nine on 1000 13.8 / 16.1 / 21.3, fp32 documents 28.1 / 27.7 / 27.5, two short ones 18.9 / 13.7 / 13.6; a bf16 chunk
  // of 64 on 1000 19.3 / 19.7 / 24.7, of 128 on 3000 31.1 / 31.1 / 30.8.
  int32_t few_chunk = 256;
  int32_t rows_chunk = 256;
  int64_t once_cells = 0;    // few rows that read at least this many cells read them past the caches (0: never)
};

// May be reused from call to call: planning a batch like the previous one allocates next to nothing.
struct ScoredPlan {
  struct Tile {  // packed rows row0 .. row0 + nrows - 1 of an entry, which see positions of [lo, hi)
    int32_t entry, row0, nrows, lo, hi;
  };
  std::vector<Extent> ext;
  std::vector<int32_t> seg_table;
  std::vector<int64_t> scratch[2];
  std::vector<Tile> few_tiles, row_tiles;
  std::vector<DkEntry> entries;  // pad[0]: the entry's prefix
  std::vector<DkSeg> segs;
  std::vector<int32_t> first;  // first position that the rows of a token see, where the call says so
  std::vector<DkItem> few, rows;
  std::vector<DkMerge> merges;
  int64_t total_tokens = 0, part_rows = 0;
  int32_t few_rows = 0, tile_rows = 0, merge_rows = 0;  // most rows of an item, of a merge
  bool merges_inside = false;                           // the kernel for few rows can merge all of them itself
  size_t off_entries = 0, off_segs = 0, off_first = 0, off_few = 0, off_rows = 0, off_merges = 0;
  size_t blob_bytes = 0, off_parts = 0, total_bytes = 0;
};

// Caller holds pool.mutex().
int32_t build_scored_plan(Pool& pool, const ScoredConfig& cfg, int32_t n_seqs, const int32_t* slots, const int32_t* cu_delta, bool staged,
                          const ScoreMasks& masks, ScoredPlan* plan);

}  // namespace dk
