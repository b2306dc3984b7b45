#include "plan_scored.hpp"

#include <algorithm>
#include <functional>

#include "plan.hpp"

namespace dk {

namespace {

typedef ScoredPlan::Tile Tile;

constexpr int64_t FEW_ROUNDS = 3;    // more rounds of workgroups even out by themselves
constexpr int64_t FIXED_KEYS = 512;  // what starting a work item and merging it cost, in keys
// Entries of few rows join the rows kernel's launch where there is one, unless they are most of the batch and come from HBM, which
// the kernel of their own reads faster.  Measured, us, on their own / joined, capped scores (K/V cells of the few; of the row tiles):
// 12 single tokens on 500-1000 beside 32 tokens (9 thousand; 1) 28.5 / 22.9, one on 6000 beside 128 (6; 24) 52.6 / 41.3, 40 sessions
// of up to 9 on 4000-8000 beside 512 (240; 96) 285 / 235, 60 on 6000-9000 beside 2 x 512 (450; 240) 481 / 467, beside 256
// (450; 60) 361 / 375, beside 32 (450; 8) 322 / 357.
constexpr int64_t JOIN_RATIO = 4;
// Most rows, and partial rows, of a merge by the last workgroup of its splits.  Merge launch / inside, us: one token on 3000 cached
// 12.2 / 10.6, on 600 11.5 / 9.9, with 64-wide heads 10.3 / 9.3, with two KV heads 11.2 / 9.8, four tokens on 2000 each 12.3 / 11.7.
constexpr int32_t INSIDE_ROWS = 8, INSIDE_PARTS = 64;

// The positions that some row of the tile sees.
void see(const ScoreMasks& masks, const DkEntry& e, int32_t group, const std::vector<int32_t>& first, Tile* t) {
  const int32_t t0 = t->row0 / group, t1 = (t->row0 + t->nrows - 1) / group;
  const auto from_of = [&](int32_t tok) { return masks.window > 0 ? std::max(0, e.n + tok - masks.window + 1) : 0; };
  t->lo = from_of(t0);
  t->hi = std::max(e.n + t1, e.pad[0] - 1) + 1;
  if (!masks.first) return;
  int32_t lo = INT32_MAX, hi = 0;
  for (int32_t tok = t0; tok <= t1; ++tok) {
    const int32_t from = std::max(from_of(tok), first[(size_t)(e.tok0 + tok)]), last = std::max(e.n + tok, e.pad[0] - 1);
    if (from > last) continue;
    lo = std::min(lo, from);
    hi = std::max(hi, last + 1);
  }
  t->lo = hi > 0 ? lo : 0;  // (rows that see nothing still get their zeros)
  t->hi = hi;
}

struct Pieces {
  int32_t n;
  int64_t keys;  // of each (the last may have fewer)
};
Pieces pieces_of(int64_t keys, int64_t chunk) {
  int64_t n = std::max<int64_t>(1, (keys + chunk - 1) / chunk);
  if (n > 1 && keys - (n - 1) * chunk < chunk / 4) --n;  // no sliver at the end
  const int64_t each = ((keys + n - 1) / n + 63) / 64 * 64;
  return {(int32_t)std::max<int64_t>(1, (keys + each - 1) / std::max<int64_t>(each, 1)), each};
}

// Keys that the busiest of `at_once` workgroups walks if the pieces are taken longest first, a start counted as `fixed` keys.
int64_t busiest(const std::vector<Tile>& tiles, int64_t chunk, int64_t fixed, int32_t at_once, std::vector<int64_t>* pieces, std::vector<int64_t>* heap) {
  pieces->clear();
  for (const Tile& t : tiles) {
    const Pieces cuts = pieces_of(t.hi - t.lo, chunk);
    for (int32_t i = 0; i < cuts.n; ++i) pieces->push_back(std::min(cuts.keys, t.hi - t.lo - i * cuts.keys) + fixed);
  }
  std::sort(pieces->begin(), pieces->end(), std::greater<int64_t>());
  heap->assign((size_t)at_once, 0);
  for (const int64_t k : *pieces) {
    std::pop_heap(heap->begin(), heap->end(), std::greater<int64_t>());
    heap->back() += k;
    std::push_heap(heap->begin(), heap->end(), std::greater<int64_t>());
  }
  return *std::max_element(heap->begin(), heap->end());
}

// Work items of tiles whose workgroups run `at_once` at a time per KV head: key ranges are cut where the longest would outlast an
// equal share, in pieces of no less than min_chunk; longest first.  Tiles that can all run at once are cut into the shortest pieces
// that still do; a few more than that, into the shortest that are done in as many rounds, if the rounds get shorter by more than the
// cuts cost.
void cut(const std::vector<Tile>& tiles, int32_t at_once, int32_t min_chunk, ScoredPlan* p, std::vector<DkItem>* items) {
  int64_t total = 0, longest = 0;
  for (const Tile& t : tiles) {
    total += t.hi - t.lo;
    longest = std::max<int64_t>(longest, t.hi - t.lo);
  }
  int64_t chunk = std::max<int64_t>(min_chunk, (total + at_once - 1) / at_once);
  chunk = (chunk + 63) / 64 * 64;
  const int64_t rounds = ((int64_t)tiles.size() + at_once - 1) / at_once;
  if (rounds >= 1 && rounds <= FEW_ROUNDS) {
    const auto fits = [&](int64_t c) {
      int64_t n = 0;
      for (const Tile& t : tiles) n += pieces_of(t.hi - t.lo, c).n;
      return n <= rounds * at_once;
    };
    int64_t least = std::max<int64_t>(min_chunk, (total + rounds * at_once - 1) / (rounds * at_once));
    least = (least + 63) / 64 * 64;
    int64_t most = std::max(least, (longest + 63) / 64 * 64);
    while (least < most) {
      const int64_t mid = (least + most) / 128 * 64;
      if (fits(mid)) most = mid;
      else least = mid + 64;
    }
    if (rounds == 1 || 10 * busiest(tiles, least, FIXED_KEYS, at_once, &p->scratch[0], &p->scratch[1]) <
                           9 * busiest(tiles, chunk, FIXED_KEYS, at_once, &p->scratch[0], &p->scratch[1]))
      chunk = least;
  }
  for (const Tile& t : tiles) {
    const int64_t keys = t.hi - t.lo;
    const Pieces cuts = pieces_of(keys, chunk);
    const int32_t ns = cuts.n;
    const int64_t each = cuts.keys;
    int32_t part0 = -1;
    if (ns > 1) {
      part0 = (int32_t)p->part_rows;
      p->part_rows += (int64_t)ns * t.nrows;
      p->merges.push_back({t.entry, t.row0, t.nrows, part0, ns, p->entries[(size_t)t.entry].tok0, {0, 0}});
      p->merge_rows = std::max(p->merge_rows, t.nrows);
    }
    for (int32_t sp = 0; sp < ns; ++sp) {
      DkItem it{};
      it.entry = t.entry;
      it.row0 = t.row0;
      it.nrows = t.nrows;
      it.kv_lo = t.lo + (int32_t)(sp * each);
      it.kv_hi = sp + 1 == ns ? t.hi : t.lo + (int32_t)((sp + 1) * each);
      it.part_row0 = ns > 1 ? part0 + sp * t.nrows : -1;
      if (ns > 1 && ns < 256 && p->merges.size() <= 256) {
        it.merge = 256 * (int32_t)(p->merges.size() - 1) + ns;
        it.part_base = part0;
      }
      items->push_back(it);
    }
  }
  std::stable_sort(items->begin(), items->end(), [](const DkItem& a, const DkItem& b) { return a.kv_hi - a.kv_lo > b.kv_hi - b.kv_lo; });
}

}  // namespace

int32_t build_scored_plan(Pool& pool, const ScoredConfig& cfg, int32_t n_seqs, const int32_t* slots, const int32_t* cu_delta, bool staged,
                          const ScoreMasks& masks, ScoredPlan* p) {
  int32_t rc = pool.check_batch(n_seqs, slots, cu_delta);
  if (rc != OK) return rc;
  p->entries.clear();
  p->segs.clear();
  p->first.clear();
  p->few_tiles.clear();
  p->row_tiles.clear();
  p->few.clear();
  p->rows.clear();
  p->merges.clear();
  p->part_rows = 0;
  p->few_rows = p->merge_rows = 0;
  p->total_tokens = n_seqs ? cu_delta[n_seqs] : 0;
  const int64_t group = cfg.n_q_heads / cfg.n_kv_heads;
  int64_t most = 0;
  for (int32_t b = 0; b < n_seqs; ++b) most = std::max<int64_t>(most, (int64_t)cu_delta[b + 1] - cu_delta[b]);
  // packed row numbers are divided by the group by a multiplication that is exact while row * (group - 1) < 2^32
  if (most >= (int64_t(1) << 31) / (group * group)) return ERR_UNSUPPORTED;
  // fp32: a compute unit has one workgroup at a time.  Items of 32 rows read K and V half as often, items of 16 take shorter rounds: 32
  // where that halves the rounds, 16 where rows have starts of their own unless there are many (32 of them see the union of more
  // documents).  Measured, us, 16 / 32 rows, a window of 200 and all of 1300 keys, by tiles of 32 rows:
  //   128  12.8 / 20.2   41 / 49      160  22.3 / 20.4   67 / 68      256  27.6 / 22.2   85 / 68      288  36.0 / 37.4  117 / 105
  //   320  36.6 / 38.4  119 / 121     384  37.2 / 42.8  124 / 129     400  45.3 / 42.9  155 / 130     512  46.5 / 43.4  166 / 137
  // and documents: 160  19.0 / 24.0, 254  24.7 / 29.6, 360  31.8 / 34.9, 400  36.6 / 34.5, 440  39.5 / 35.8.
  const int64_t tiles = (p->total_tokens * group + 31) / 32 * cfg.n_kv_heads;
  const bool halves = tiles > 384 || (tiles > 128 && tiles <= 256 && !masks.first);
  p->tile_rows = cfg.bf16 ? 128 : halves ? 32 : 16;
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
    if (masks.first) {
      for (int32_t t = 0; t < delta; ++t) {
        const int64_t f = masks.first[cu_delta[b] + t];
        if (f < 0) return ERR_INVALID;
        p->first.push_back((int32_t)std::min<int64_t>(f, INT32_MAX / 2));
      }
    }
    const int32_t rows = (int32_t)group * delta;
    const bool few = cfg.bf16 && rows <= cfg.few_rows;
    const int32_t step = few ? cfg.few_rows : p->tile_rows;
    if (few) p->few_rows = std::max(p->few_rows, rows);
    for (int32_t r0 = 0; r0 < rows; r0 += step) {
      Tile t{b, r0, std::min(step, rows - r0), 0, 0};
      see(masks, e, (int32_t)group, p->first, &t);
      (few ? p->few_tiles : p->row_tiles).push_back(t);
    }
  }
  int64_t cells = 0, row_cells = 0;
  for (const Tile& t : p->few_tiles) cells += t.hi - t.lo;
  for (const Tile& t : p->row_tiles) row_cells += t.hi - t.lo;
  if (!p->row_tiles.empty() && (cells < cfg.once_cells || cells <= JOIN_RATIO * row_cells)) {
    p->row_tiles.insert(p->row_tiles.end(), p->few_tiles.begin(), p->few_tiles.end());
    p->few_tiles.clear();
    p->few_rows = 0;
    cells = 0;
  }
  // (64 verifying sessions of 4096 visible keys, 1.08 GB: 210 us through the caches, 190 past them.)
  if (cells >= cfg.once_cells) mark_unshared(&p->segs, &p->seg_table, cfg.once_cells);
  cut(p->few_tiles, std::max(1, 256 / cfg.n_kv_heads), cfg.few_chunk, p, &p->few);
  cut(p->row_tiles, std::max(1, (cfg.bf16 ? 512 : 256) / cfg.n_kv_heads), cfg.rows_chunk, p, &p->rows);
  // Merging inside the kernel for few rows, under the streaming kernel's conditions (see merges_inside there).
  // (Its form for more than 32 rows does not.)
  p->merges_inside = p->rows.empty() && p->few_rows <= 32 && !p->merges.empty() &&
                     p->merges.size() * (size_t)cfg.n_kv_heads <= (size_t)ARRIVALS_PER_SLICE;
  for (const DkMerge& m : p->merges) p->merges_inside &= m.nrows <= INSIDE_ROWS && m.nsplit * m.nrows <= INSIDE_PARTS && m.nsplit < 256;
  const auto section = [](size_t& at, size_t bytes) {
    const size_t off = at;
    at = (at + bytes + 15) / 16 * 16;
    return off;
  };
  size_t at = 0;
  p->off_entries = section(at, p->entries.size() * sizeof(DkEntry));
  p->off_segs = section(at, p->segs.size() * sizeof(DkSeg));
  p->off_few = section(at, p->few.size() * sizeof(DkItem));
  p->off_rows = section(at, p->rows.size() * sizeof(DkItem));
  p->off_merges = section(at, p->merges.size() * sizeof(DkMerge));
  p->off_first = section(at, p->first.size() * sizeof(int32_t));
  p->blob_bytes = at;
  p->off_parts = (at + 255) / 256 * 256;
  p->total_bytes = p->off_parts + (size_t)p->part_rows * cfg.n_kv_heads * (cfg.head_dim + 2) * sizeof(float) + 256;
  return OK;
}

}  // namespace dk
