#include "plan_scored.hpp"

#include <algorithm>

namespace dk {

int32_t build_scored_plan(Pool& pool, int32_t n_seqs, const int32_t* slots, const int32_t* cu_delta, bool staged,
                          const ScoreMasks& masks, ScoredPlan* p) {
  int32_t rc = pool.check_batch(n_seqs, slots, cu_delta);
  if (rc != OK) return rc;
  p->entries.clear();
  p->segs.clear();
  p->first.clear();
  p->total_tokens = n_seqs ? cu_delta[n_seqs] : 0;
  for (int32_t b = 0; b < n_seqs; ++b) {
    const int32_t delta = cu_delta[b + 1] - cu_delta[b];
    int64_t len = 0;
    rc = pool.extents_locked(slots[b], &p->ext, &len);
    if (rc != OK) return rc;
    if (!staged && delta > len) return ERR_INVALID;
    if (len + delta > INT32_MAX / 2) return ERR_UNSUPPORTED;
    if (masks.prefix && masks.prefix[b] < 0) return ERR_INVALID;
    DkEntry e{};
    e.seg_begin = (int32_t)p->segs.size();
    e.n = (int32_t)(staged ? len : len - delta);
    e.delta = delta;
    e.tok0 = cu_delta[b];
    e.pad[0] = masks.prefix ? (int32_t)std::min<int64_t>(masks.prefix[b], e.n + delta) : 0;
    if (delta > 0) {
      for (const Extent& x : p->ext) p->segs.push_back({x.cell, (int32_t)x.pos, (int32_t)x.len, 0, 0});
      if (staged) p->segs.push_back({(int64_t)cu_delta[b], e.n, delta, 1, 0});
    }
    e.seg_end = (int32_t)p->segs.size();
    p->entries.push_back(e);
    if (!masks.first) continue;
    for (int32_t t = 0; t < delta; ++t) {
      const int64_t f = masks.first[cu_delta[b] + t];
      if (f < 0) return ERR_INVALID;
      p->first.push_back((int32_t)std::min<int64_t>(f, INT32_MAX / 2));
    }
  }
  const auto section = [](size_t& at, size_t bytes) {
    const size_t off = at;
    at = (at + bytes + 15) / 16 * 16;
    return off;
  };
  size_t at = 0;
  p->off_entries = section(at, p->entries.size() * sizeof(DkEntry));
  p->off_segs = section(at, p->segs.size() * sizeof(DkSeg));
  p->off_first = section(at, p->first.size() * sizeof(int32_t));
  p->blob_bytes = at;
  p->total_bytes = (at + 255) / 256 * 256 + 256;
  return OK;
}

}  // namespace dk
