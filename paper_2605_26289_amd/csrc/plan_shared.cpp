#include "plan_shared.hpp"

#include <algorithm>
#include <cmath>

namespace dk {

namespace {

// What the cuts go by: microseconds of a workgroup's place, of which the chip has 512 (fp32: 256).  Measured by clocks in the kernels.
constexpr double FIXED_US = 6.0, F32_FIXED_US = 8.0;  // a work item without its keys
constexpr double ROWS_KEY_US = 2.3 / 64;  // a key of a tile of 128 rows of 128
constexpr double FEW_KEY_US = 1.9 / 64;   // a key of a tile of up to 32 rows
constexpr double FEW2_KEY_US = 2.6 / 64;  // a key of one of up to 64
constexpr double F32_KEY_US = 2.5 / 64;   // a key of 32 rows of 128 in fp32
constexpr double PART_US = 0.08;          // a partial row of 128, written and read

double places(const SharedConfig& cfg) { return std::max(1.0, (cfg.bf16 ? 512.0 : 256.0) / cfg.n_kv_heads); }  // of a KV head
double fixed_us(const SharedConfig& cfg) { return cfg.bf16 ? FIXED_US : F32_FIXED_US; }
double key_us(const SharedConfig& cfg, int64_t rows) {
  const double width = 0.2 + 0.8 * cfg.head_dim / 128;
  if (!cfg.bf16) return F32_KEY_US * width;
  return (rows <= 32 ? FEW_KEY_US : rows <= SHARED_FEW ? FEW2_KEY_US : ROWS_KEY_US) * width;
}
double part_us(const SharedConfig& cfg) { return PART_US * cfg.head_dim / 128; }
int64_t tile_rows(const SharedConfig& cfg, const SharedPlan& p, int64_t rows) {
  if (!cfg.bf16) return p.tile_rows;
  return rows <= SHARED_FEW ? SHARED_FEW : SHARED_TILE;
}
double tiles_us(const SharedConfig& cfg, const SharedPlan& p, int64_t rows) {  // a key for all rows
  const int64_t tile = tile_rows(cfg, p, rows);
  return key_us(cfg, rows) * (double)((rows + tile - 1) / tile);
}

struct Builder {
  const SharedConfig& cfg;
  const int32_t* cu;
  bool staged;
  SharedPlan* p;
  int64_t group;

  int64_t rows_of(int32_t entry) const { return (int64_t)(cu[entry + 1] - cu[entry]) * group; }
  // Segments of positions [lo, hi) of an entry's cells.
  void add_segs(int32_t entry, int64_t lo, int64_t hi) {
    p->ext.clear();
    for (int32_t i = p->part0[(size_t)entry]; i < p->part0[(size_t)entry + 1]; ++i) {
      const Pool::Part& x = p->parts[(size_t)i];
      if (std::max(lo, x.lo) < std::min(hi, x.hi)) Pool::add_extents(*x.node, std::max(lo, x.lo), std::min(hi, x.hi), &p->ext);
    }
    for (const Extent& x : p->ext) p->node_segs.push_back({(int32_t)x.cell, (int32_t)x.pos, (int32_t)x.len});
  }

  // Whether the members' rows together over `keys` positions cost less than each entry's alone.
  bool worth_sharing(int32_t begin, int32_t end, int64_t keys) const {
    double alone = 0.0;
    int64_t rows = 0;
    for (int32_t i = begin; i < end; ++i) {
      const int64_t r = rows_of(p->members[(size_t)i].entry);
      rows += r;
      alone += tiles_us(cfg, *p, r);
    }
    const double together = tiles_us(cfg, *p, rows), tiles = together / key_us(cfg, rows);
    const double pieces = std::max(1.0, std::min((double)keys / 512.0, places(cfg) / tiles));
    return (double)keys * (alone - together) > fixed_us(cfg) + part_us(cfg) * pieces * (double)rows;
  }

  void add_own(const SharedPlan::Member& m, int64_t start) {
    const int32_t b = m.entry, delta = cu[b + 1] - cu[b];
    const int64_t n = p->n[(size_t)b];
    SharedPlan::Node x{};
    x.entry = b;
    x.link = m.link;
    x.seg0 = (int32_t)p->node_segs.size();
    add_segs(b, start, staged ? n : n + delta);
    if (staged) p->node_segs.push_back({~cu[b], (int32_t)n, delta});
    x.nsegs = (int32_t)p->node_segs.size() - x.seg0;
    x.d = {cu[b], (int32_t)rows_of(b), (int32_t)start, (int32_t)(n + delta - start), 0, 0, -1, (int32_t)n};
    p->nodes.push_back(x);
  }

  void add_shared(int32_t begin, int32_t end, int64_t start, int64_t pos) {
    SharedPlan::Node x{};
    x.entry = x.link = -1;
    x.seg0 = (int32_t)p->node_segs.size();
    add_segs(p->members[(size_t)begin].entry, start, pos);
    x.nsegs = (int32_t)p->node_segs.size() - x.seg0;
    const int32_t tok0 = (int32_t)p->tokens.size();
    int64_t rows = 0;
    for (int32_t i = begin; i < end; ++i) {
      SharedPlan::Member& m = p->members[(size_t)i];
      p->links.push_back({(int32_t)p->nodes.size(), (int32_t)rows, m.link});
      m.link = (int32_t)p->links.size() - 1;
      for (int32_t t = cu[m.entry]; t < cu[m.entry + 1]; ++t) p->tokens.push_back(t);
      rows += rows_of(m.entry);
    }
    x.d = {tok0, (int32_t)rows, (int32_t)start, (int32_t)(pos - start), 0, 0, 0, SHARED_ALL};
    p->nodes.push_back(x);
  }

  // The tree of shared prefixes, from the roots down: members that have a position in the same node of the pool stay together.
  void build() {
    p->tasks.clear();
    if (!p->members.empty()) p->tasks.push_back({0, (int32_t)p->members.size(), 0, 0});
    while (!p->tasks.empty()) {
      SharedPlan::Task t = p->tasks.back();
      p->tasks.pop_back();
      if (t.end - t.begin == 1) {
        add_own(p->members[(size_t)t.begin], t.start);
        continue;
      }
      while (true) {  // as far as all of them have the same cells
        int64_t step = INT64_MAX;
        const Node* same = nullptr;
        for (int32_t i = t.begin; i < t.end && step > 0; ++i) {
          SharedPlan::Member& m = p->members[(size_t)i];
          if (p->n[(size_t)m.entry] <= t.pos) {
            step = 0;
            break;
          }
          while (p->parts[(size_t)m.part].hi <= t.pos) ++m.part;
          const Pool::Part& x = p->parts[(size_t)m.part];
          if (same && x.node != same) step = 0;
          same = x.node;
          step = std::min(step, std::min(x.hi, p->n[(size_t)m.entry]) - t.pos);
        }
        if (step <= 0) break;
        t.pos += step;
      }
      if (t.pos > t.start && worth_sharing(t.begin, t.end, t.pos - t.start)) {
        add_shared(t.begin, t.end, t.start, t.pos);
        t.start = t.pos;
      }
      // those that end here part from all others, the rest by the node they go on in
      for (int32_t i = t.begin; i < t.end; ++i) {
        SharedPlan::Member& m = p->members[(size_t)i];
        if (p->n[(size_t)m.entry] <= t.pos) {
          m.key = -1 - i;
          continue;
        }
        while (p->parts[(size_t)m.part].hi <= t.pos) ++m.part;
        m.key = p->parts[(size_t)m.part].node->cell_of(0);
      }
      std::sort(p->members.begin() + t.begin, p->members.begin() + t.end, [](const SharedPlan::Member& a, const SharedPlan::Member& b) {
        return a.key != b.key ? a.key < b.key : a.entry < b.entry;
      });
      for (int32_t i = t.begin; i < t.end;) {
        int32_t j = i + 1;
        while (j < t.end && p->members[(size_t)j].key == p->members[(size_t)i].key) ++j;
        p->tasks.push_back({i, j, t.start, t.pos});
        i = j;
      }
    }
  }

  // Pieces of what takes keys_us, items of at most `us` (and of 128 keys and more).
  int64_t pieces_of(double keys_us, double per_key, double us) const {
    const double most = std::max(us - fixed_us(cfg), 128 * per_key);
    return keys_us <= most ? 1 : (int64_t)(keys_us / most * 0.999) + 1;
  }
  int64_t chunk_of(const SharedPlan::Node& x, double us) const {
    const int64_t step = cfg.bf16 ? 64 : 128;  // keys that all wavefronts of an item take at a time
    const int64_t pieces = pieces_of(x.per_key * x.d.keys, x.per_key, us);
    return pieces == 1 ? (x.d.keys + 63) / 64 * 64 : ((x.d.keys + pieces - 1) / pieces + step - 1) / step * step;
  }

  // `n` items of the same length go where places are free first; `levels`: when how many places are free, soonest first.
  void put_items(double n, double us) {
    std::vector<SharedPlan::Level>& at = p->levels;
    while (n > 0) {
      const double k = std::min(n, at[0].places), end = 0.5 * (double)((int64_t)(2 * (at[0].us + us)) + 1);  // (half microseconds: few levels)
      n -= k;
      at[0].places -= k;
      size_t i = at[0].places > 0 ? 0 : 1;
      const size_t gone = i;
      while (i < at.size() && at[i].us < end) ++i;
      if (i < at.size() && at[i].us == end) at[i].places += k;
      else at.insert(at.begin() + (std::ptrdiff_t)i, {end, k});
      if (gone) at.erase(at.begin());
    }
  }

  // The longest time that a work item may take, so that all are done soonest: as long as the longest where they all run at once; else
  // until the last of those that are cut are done, longest first, or the mean of the places' loads and half of the longest of the others;
  // and the partial rows' way to memory and back.
  void choose_pieces() {
    const double at_once = places(cfg), fixed = fixed_us(cfg);
    std::vector<SharedPlan::Load>& loads = p->loads;  // longest first: only those before the first that fits are cut
    loads.clear();
    for (const SharedPlan::Node& x : p->nodes)
      loads.push_back({fixed + x.per_key * x.d.keys, x.per_key, (double)x.tiles, (double)x.d.rows, x.entry < 0 || x.link >= 0 ? 1.0 : 0.0, 1, 0});
    std::sort(loads.begin(), loads.end(), [](const SharedPlan::Load& a, const SharedPlan::Load& b) { return a.us > b.us; });
    double all = 0, items = 0, parts = 0;  // of those that are not cut
    for (const SharedPlan::Load& x : loads) {
      all += x.tiles * x.us;
      items += x.tiles;
      parts += x.part * x.rows;
    }
    const double least = fixed * 1.2;
    double best_us = loads[0].us, best = 1e300;
    size_t n_cut = 0;
    for (double us = loads[0].us; us > least; us *= 0.9) {
      for (; n_cut < loads.size() && loads[n_cut].us > us; ++n_cut) {
        const SharedPlan::Load& x = loads[n_cut];
        all -= x.tiles * x.us;
        items -= x.tiles;
        parts -= x.part * x.rows;
      }
      const double uncut = n_cut < loads.size() ? loads[n_cut].us : 0;
      double longest = uncut, cut_all = 0, cut_items = 0, cut_parts = 0;
      for (size_t i = 0; i < n_cut; ++i) {
        SharedPlan::Load& x = loads[i];
        const double keys_us = x.us - fixed;
        x.pieces = (double)pieces_of(keys_us, x.per_key, us);
        x.piece_us = fixed + keys_us / x.pieces;
        longest = std::max(longest, x.piece_us);
        cut_all += x.tiles * (x.pieces * fixed + keys_us);
        cut_items += x.tiles * x.pieces;
        cut_parts += x.pieces * x.rows;
      }
      const double joined = part_us(cfg) * (parts + cut_parts) / at_once + (parts + cut_parts > 0 ? 3.0 : 0.0);
      const double mean = (all + cut_all) / at_once;
      if (mean + joined >= best) break;  // shorter items only add to both
      double run = longest;
      if (items + cut_items > 16 * at_once) {
        run = mean + 0.5 * longest;
      } else if (items + cut_items > at_once) {
        p->levels.assign(1, {0, at_once});
        for (size_t i = 0; i < n_cut; ++i) put_items(loads[i].tiles * loads[i].pieces, loads[i].piece_us);
        run = std::max(p->levels.back().us, mean + 0.5 * uncut);
      }
      const double est = run + joined;
      if (est < best) {
        best = est;
        best_us = us;
      }
      if (items + cut_items > 16 * at_once) break;
    }
    for (SharedPlan::Node& x : p->nodes) {
      x.d.chunk = (int32_t)chunk_of(x, best_us);
      x.pieces = (x.d.keys + x.d.chunk - 1) / x.d.chunk;
    }
  }
};

size_t section(size_t& at, size_t bytes) {
  const size_t off = at;
  at = (at + bytes + 15) / 16 * 16;
  return off;
}

}  // namespace

int32_t build_shared_plan(Pool& pool, const SharedConfig& cfg, int32_t n_seqs, const int32_t* slots, const int32_t* cu_delta, bool staged,
                          SharedPlan* p) {
  int32_t rc = pool.check_batch(n_seqs, slots, cu_delta);
  if (rc != OK) return rc;
  p->parts.clear();
  p->part0.clear();
  p->n.clear();
  p->members.clear();
  p->links.clear();
  p->nodes.clear();
  p->node_segs.clear();
  p->starts.clear();
  p->out_nodes.clear();
  p->segs.clear();
  p->tokens.clear();
  p->blocks.clear();
  p->src0.clear();
  p->sources.clear();
  p->total_tokens = n_seqs ? cu_delta[n_seqs] : 0;
  p->part_rows = p->items = p->row_items = 0;
  const int64_t group = cfg.n_q_heads / cfg.n_kv_heads;
  // packed row numbers are divided by the group by a multiplication that is exact while row * (group - 1) < 2^32
  if (p->total_tokens >= (int64_t(1) << 31) / (group * group)) return ERR_UNSUPPORTED;
  p->tile_rows = p->total_tokens * group <= 16 ? 16 : 32;
  for (int32_t b = 0; b < n_seqs; ++b) {
    const int32_t delta = cu_delta[b + 1] - cu_delta[b];
    int64_t len = 0;
    p->part0.push_back((int32_t)p->parts.size());
    rc = pool.chain_locked(slots[b], &p->parts, &len);
    if (rc != OK) return rc;
    if (!staged && delta > len) return ERR_INVALID;
    if (len + delta >= SHARED_ALL / 2) return ERR_UNSUPPORTED;
    p->n.push_back(staged ? len : len - delta);
    if (delta == 0) continue;
    p->members.push_back({b, p->part0.back(), -1, 0});
  }
  p->part0.push_back((int32_t)p->parts.size());
  Builder build{cfg, cu_delta, staged, p, group};
  build.build();
  for (SharedPlan::Node& x : p->nodes) {
    const int64_t tile = tile_rows(cfg, *p, x.d.rows);
    x.tiles = (int32_t)((x.d.rows + tile - 1) / tile);
    x.per_key = (float)key_us(cfg, x.d.rows);
  }
  if (!p->nodes.empty()) build.choose_pieces();
  // longest items first
  p->order.resize(p->nodes.size());
  for (size_t i = 0; i < p->nodes.size(); ++i) {
    p->order[i] = (int32_t)i;
    SharedPlan::Node& x = p->nodes[i];
    x.fixed = x.per_key * (float)std::min(x.d.chunk, x.d.keys);
    if (x.entry < 0 || x.link >= 0 || x.pieces > 1) {
      x.d.part0 = (int32_t)p->part_rows;
      p->part_rows += (int64_t)x.pieces * x.d.rows;
      if (p->part_rows > INT32_MAX / 2) return ERR_UNSUPPORTED;
    }
  }
  std::stable_sort(p->order.begin(), p->order.end(), [&](int32_t a, int32_t b) { return p->nodes[(size_t)a].fixed > p->nodes[(size_t)b].fixed; });
  for (const int32_t i : p->order) {
    SharedPlan::Node& x = p->nodes[(size_t)i];
    x.d.seg0 = (int32_t)p->segs.size();
    p->segs.insert(p->segs.end(), p->node_segs.begin() + x.seg0, p->node_segs.begin() + x.seg0 + x.nsegs);
    p->starts.push_back((int32_t)p->items);
    p->out_nodes.push_back(x.d);
    p->items += (int64_t)x.tiles * x.pieces;
    if (x.d.rows > SHARED_FEW) p->row_items += (int64_t)x.tiles * x.pieces;
    if (p->items > INT32_MAX / 64 / cfg.n_kv_heads) return ERR_UNSUPPORTED;
  }
  p->starts.push_back((int32_t)p->items);
  DkShNode last{};
  last.seg0 = (int32_t)p->segs.size();
  p->out_nodes.push_back(last);
  // merges: the rows of entries that have more than one partial row
  int64_t merge_rows = 0, most = 0;
  p->n_merges = 0;
  for (const int32_t i : p->order) {
    const SharedPlan::Node& x = p->nodes[(size_t)i];
    p->src0.push_back((int32_t)p->sources.size());
    if (x.entry < 0 || x.d.part0 < 0) continue;
    ++p->n_merges;
    merge_rows += x.d.rows;
    int64_t all = x.pieces;
    for (int32_t l = x.link; l >= 0; l = p->links[(size_t)l].before) {
      const SharedPlan::Link& k = p->links[(size_t)l];
      const SharedPlan::Node& y = p->nodes[(size_t)k.node];
      p->sources.push_back({y.d.part0 + k.row0, y.d.rows, y.pieces});
      all += y.pieces;
    }
    most = std::max(most, all);
  }
  p->src0.push_back((int32_t)p->sources.size());
  // Lane groups share the partial rows of a row where there are too few rows to fill the chip otherwise.
  const int64_t groups = 1024 / cfg.head_dim;
  p->spread = 1;
  while (p->spread < groups && 2 * p->spread <= most && merge_rows * cfg.n_kv_heads * p->spread < 8192) p->spread *= 2;
  const int64_t rows_a_block = groups / p->spread;
  int64_t blocks = 0;
  for (const int32_t i : p->order) {
    const SharedPlan::Node& x = p->nodes[(size_t)i];
    p->blocks.push_back((int32_t)std::min<int64_t>(blocks, INT32_MAX));
    if (x.entry >= 0 && x.d.part0 >= 0) blocks += (x.d.rows + rows_a_block - 1) / rows_a_block;
  }
  if (blocks > INT32_MAX / 256 / cfg.n_kv_heads) return ERR_UNSUPPORTED;
  p->merge_blocks = (int32_t)blocks;
  p->blocks.push_back((int32_t)blocks);
  size_t at = 0;
  section(at, p->starts.size() * sizeof(int32_t));
  p->off_nodes = section(at, p->out_nodes.size() * sizeof(DkShNode));
  p->off_segs = section(at, p->segs.size() * sizeof(DkShSeg));
  p->off_tokens = section(at, p->tokens.size() * sizeof(int32_t));
  p->main_bytes = at;
  at = 0;
  section(at, p->blocks.size() * sizeof(int32_t));
  p->off_src0 = section(at, p->src0.size() * sizeof(int32_t));
  p->off_sources = section(at, p->sources.size() * sizeof(DkShSource));
  p->merge_bytes = at;
  p->off_merge = p->main_bytes;
  p->off_parts = (p->main_bytes + p->merge_bytes + 255) / 256 * 256;
  p->total_bytes = p->off_parts + (size_t)p->part_rows * cfg.n_kv_heads * (cfg.head_dim + 2) * sizeof(float) + 256;
  return OK;
}

}  // namespace dk
