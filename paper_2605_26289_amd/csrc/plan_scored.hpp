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

// May be reused from call to call: planning a batch like the previous one allocates next to nothing.
struct ScoredPlan {
  std::vector<Extent> ext;
  std::vector<DkEntry> entries;  // pad[0]: the entry's prefix
  std::vector<DkSeg> segs;
  std::vector<int32_t> first;  // first position that the rows of a token see, where the call says so
  int64_t total_tokens = 0;
  size_t off_entries = 0, off_segs = 0, off_first = 0;
  size_t blob_bytes = 0, total_bytes = 0;
};

// Caller holds pool.mutex().
int32_t build_scored_plan(Pool& pool, int32_t n_seqs, const int32_t* slots, const int32_t* cu_delta, bool staged,
                          const ScoreMasks& masks, ScoredPlan* plan);

}  // namespace dk
