// Checks plans of attention for batches that share cells against the definition, on seeded pools: every (row, position) pair in exactly
// one work item, through the entry's own cells; partial rows disjoint; the merge finds exactly the pieces that were written.
#include <algorithm>
#include <cstdio>
#include <cstdlib>
#include <map>
#include <random>
#include <set>
#include <vector>

#include "../paper_2605_26289_amd/csrc/plan_shared.hpp"

using namespace dk;

#define CHECK(x)                                                       \
  do {                                                                 \
    if (!(x)) {                                                        \
      std::printf("FAILED line %d: %s (seed %d)\n", __LINE__, #x, g_seed); \
      std::exit(1);                                                    \
    }                                                                  \
  } while (0)
static int g_seed = 0;

struct Shape {
  int hq, hkv, d;
  bool bf16;
};

static int64_t g_shared = 0, g_pieces = 0, g_inline = 0, g_carried = 0, g_direct = 0;

static void check(Pool& pool, const Shape& sh, const std::vector<int32_t>& slots, const std::vector<int32_t>& cu, bool staged) {
  SharedConfig cfg;
  cfg.n_q_heads = sh.hq;
  cfg.n_kv_heads = sh.hkv;
  cfg.head_dim = sh.d;
  cfg.bf16 = sh.bf16;
  static SharedPlan p;  // reused, as a pool does
  CHECK(build_shared_plan(pool, cfg, (int32_t)slots.size(), slots.data(), cu.data(), staged, &p) == OK);
  const int group = sh.hq / sh.hkv;
  const int n_nodes = (int)p.out_nodes.size() - 1;
  CHECK((int)p.starts.size() == n_nodes + 1 && p.starts[n_nodes] == p.items);
  if (p.total_tokens == 0) {
    CHECK(n_nodes == 0 && p.n_merges == 0);
    return;
  }
  (p.in_args() ? g_inline : g_carried)++;
  CHECK(!p.in_args() || p.merge_in_args());
  // sections fit one behind the other
  CHECK(p.starts.size() * 4 <= p.off_nodes && p.off_nodes + p.out_nodes.size() * sizeof(DkShNode) <= p.off_segs);
  CHECK(p.off_segs + p.segs.size() * sizeof(DkShSeg) <= p.off_tokens && p.off_tokens + p.tokens.size() * 4 <= p.main_bytes);
  CHECK((int)p.blocks.size() == n_nodes + 1 && (int)p.src0.size() == n_nodes + 1);
  CHECK(p.blocks.size() * 4 <= p.off_src0 && p.off_src0 + p.src0.size() * 4 <= p.off_sources && p.off_sources + p.sources.size() * sizeof(DkShSource) <= p.merge_bytes);
  CHECK(p.off_merge == p.main_bytes && p.off_merge + p.merge_bytes <= p.off_parts);
  CHECK(p.off_parts + (size_t)p.part_rows * sh.hkv * (sh.d + 2) * 4 <= p.total_bytes);

  // what every packed token sees: cells by position (staged rows: negative numbers)
  const int64_t tokens = p.total_tokens;
  std::vector<std::vector<int64_t>> cells((size_t)slots.size());
  std::vector<int> entry_of((size_t)tokens);
  std::vector<int64_t> limit((size_t)tokens);
  for (size_t b = 0; b < slots.size(); ++b) {
    int64_t len = 0;
    CHECK(pool.length(slots[b], &len) == OK);
    cells[b].resize((size_t)len);
    CHECK(pool.cells(slots[b], cells[b].data(), len) == OK);
    const int delta = cu[b + 1] - cu[b];
    const int64_t n = staged ? len : len - delta;
    if (staged)
      for (int t = cu[b]; t < cu[b + 1]; ++t) cells[b].push_back(~(int64_t)t);
    for (int t = cu[b]; t < cu[b + 1]; ++t) {
      entry_of[(size_t)t] = (int)b;
      limit[(size_t)t] = n + t - cu[b];
    }
  }
  const int64_t rows = tokens * group;
  std::vector<std::vector<std::pair<int64_t, int64_t>>> seen((size_t)rows);  // ranges of positions by packed row
  std::vector<int64_t> owner((size_t)p.part_rows, -1);                          // packed row whose sums a partial row holds
  std::vector<char> direct((size_t)rows, 0);
  for (int i = 0; i < n_nodes; ++i) {
    const DkShNode& nd = p.out_nodes[(size_t)i];
    CHECK(nd.rows > 0 && nd.keys > 0 && nd.chunk > 0 && nd.chunk % 64 == 0 && nd.rows % group == 0);
    CHECK(p.starts[(size_t)i] < p.starts[(size_t)i + 1]);
    const int seg_end = p.out_nodes[(size_t)i + 1].seg0;
    CHECK(nd.seg0 < seg_end && p.segs[(size_t)nd.seg0].pos == nd.lo);
    for (int s = nd.seg0; s + 1 < seg_end; ++s) CHECK(p.segs[(size_t)s].pos + p.segs[(size_t)s].len == p.segs[(size_t)s + 1].pos);
    CHECK(p.segs[(size_t)seg_end - 1].pos + p.segs[(size_t)seg_end - 1].len == nd.lo + nd.keys);
    const int tile = !sh.bf16 ? p.tile_rows : nd.rows <= SHARED_FEW ? SHARED_FEW : SHARED_TILE;
    const int tiles = (nd.rows + tile - 1) / tile;
    const int items = p.starts[(size_t)i + 1] - p.starts[(size_t)i];
    CHECK(items % tiles == 0);
    g_shared += nd.n == SHARED_ALL;
    g_pieces += items / tiles;
    for (int u = 0; u < items; ++u) {
      const int piece = u / tiles, row0 = (u - piece * tiles) * tile, nrows = std::min(tile, nd.rows - row0);
      const int64_t lo = nd.lo + (int64_t)piece * nd.chunk;
      const int64_t hi = std::min<int64_t>(std::min<int64_t>(nd.lo + nd.keys, lo + nd.chunk), (int64_t)nd.n + (row0 + nrows - 1) / group + 1);
      if (nd.part0 < 0) CHECK(piece == 0 && nd.n != SHARED_ALL);
      if (lo >= hi) {
        CHECK(piece > 0);
        continue;
      }
      for (int r = row0; r < row0 + nrows; ++r) {
        const int tok = nd.n == SHARED_ALL ? p.tokens[(size_t)(nd.tok0 + r / group)] : nd.tok0 + r / group;
        CHECK(tok >= 0 && tok < tokens);
        const int64_t row = (int64_t)tok * group + r % group;
        const int64_t last = std::min<int64_t>(hi, limit[(size_t)tok] + 1);
        if (nd.n == SHARED_ALL) CHECK(limit[(size_t)tok] >= hi - 1);
        else CHECK((int64_t)nd.n + r / group == limit[(size_t)tok]);
        if (lo < last) seen[(size_t)row].push_back({lo, last});
        if (nd.part0 >= 0) {
          const int64_t part = nd.part0 + (int64_t)piece * nd.rows + r;
          CHECK(part < p.part_rows && owner[(size_t)part] == -1);
          owner[(size_t)part] = row;
        } else {
          CHECK(!direct[(size_t)row]);
          direct[(size_t)row] = 1;
          ++g_direct;
        }
        // the cells are the entry's own
        const std::vector<int64_t>& own = cells[(size_t)entry_of[(size_t)tok]];
        if (r % group == 0)
          for (int s = nd.seg0; s < seg_end; ++s) {
            const DkShSeg& sg = p.segs[(size_t)s];
            for (int64_t at : {(int64_t)sg.pos, (int64_t)sg.pos + sg.len - 1}) {
              const int64_t cell = sg.start >= 0 ? sg.start + at - sg.pos : ~((int64_t)~sg.start + at - sg.pos);
              CHECK(at < (int64_t)own.size() && own[(size_t)at] == cell);
            }
          }
      }
    }
  }
  for (int64_t row = 0; row < rows; ++row) {
    std::vector<std::pair<int64_t, int64_t>>& v = seen[(size_t)row];
    std::sort(v.begin(), v.end());
    int64_t at = 0;
    for (const auto& r : v) {
      CHECK(r.first == at);
      at = r.second;
    }
    CHECK(at == limit[(size_t)(row / group)] + 1);
  }
  // merges: every partial row that was written is taken once, for its own row
  std::vector<char> merged((size_t)rows, 0);
  int64_t taken = 0, written = 0;
  for (int64_t o : owner) written += o >= 0;
  const int tile_rows = sh.bf16 ? SHARED_TILE : p.tile_rows;
  const int rows_a_block = 1024 / sh.d / p.spread;
  CHECK(p.spread >= 1 && rows_a_block >= 1 && (p.spread & (p.spread - 1)) == 0);
  int n_merges = 0;
  for (int i = 0; i < n_nodes; ++i) {
    const DkShNode& m = p.out_nodes[(size_t)i];
    const int n_blocks = p.blocks[(size_t)i + 1] - p.blocks[(size_t)i];
    if (m.n == SHARED_ALL || m.part0 < 0) {
      CHECK(n_blocks == 0 && p.src0[(size_t)i] == p.src0[(size_t)i + 1]);
      continue;
    }
    ++n_merges;
    CHECK(n_blocks == (m.rows + rows_a_block - 1) / rows_a_block);
    for (int r = 0; r < m.rows; ++r) {
      const int64_t row = (int64_t)m.tok0 * group + r;
      CHECK(!merged[(size_t)row] && !direct[(size_t)row]);
      merged[(size_t)row] = 1;
      const int tile_last = (std::min(m.rows, (r / tile_rows + 1) * tile_rows) - 1) / group;
      const int own = (int)((std::min<int64_t>(m.keys, (int64_t)m.n + 1 - m.lo + tile_last) + m.chunk - 1) / m.chunk);
      CHECK(own >= 1);
      for (int k = 0; k < own; ++k, ++taken) CHECK(owner[(size_t)(m.part0 + (int64_t)k * m.rows + r)] == row);
      for (int s = p.src0[(size_t)i]; s < p.src0[(size_t)i + 1]; ++s)
        for (int k = 0; k < p.sources[(size_t)s].pieces; ++k, ++taken)
          CHECK(owner[(size_t)(p.sources[(size_t)s].part0 + (int64_t)k * p.sources[(size_t)s].step + r)] == row);
    }
  }
  CHECK(p.blocks.back() == p.merge_blocks && taken == written && n_merges == p.n_merges);
  for (int64_t row = 0; row < rows; ++row) CHECK(merged[(size_t)row] + direct[(size_t)row] == 1);
}

int main(int argc, char** argv) {
  const int seeds = argc > 1 ? std::atoi(argv[1]) : 300;
  const Shape shapes[] = {{32, 8, 128, true}, {8, 2, 64, true}, {7, 1, 64, true}, {12, 2, 128, true}, {4, 4, 128, true}, {16, 1, 128, true}, {4, 1, 64, false}, {8, 2, 128, false}};
  for (int seed = 0; seed < seeds; ++seed) {
    g_seed = seed;
    std::mt19937 rng(seed);
    const auto below = [&](int n) { return (int)(rng() % (unsigned)std::max(1, n)); };
    const Shape& sh = shapes[seed % 8];
    const int granule = 1 << (4 + below(5));
    Pool pool(160, 0, 1 << 22, granule);
    std::vector<int32_t> all;
    const auto fresh = [&]() {
      int32_t s = -1;
      CHECK(pool.acquire(0, 0, &s) == OK);
      all.push_back(s);
      return s;
    };
    const auto grow = [&](int32_t s, int n) {
      const int32_t c[2] = {0, n};
      CHECK(pool.append(1, &s, c, nullptr, nullptr) == OK);
    };
    const int roots = 1 + below(4), members = 1 + below(seed % 10 == 0 ? 100 : 24);
    const int longest = seed % 3 == 0 ? 20000 : seed % 3 == 1 ? 2000 : 100;
    for (int i = 0; i < roots; ++i) grow(fresh(), 1 + below(longest));
    for (int i = 0; i < members; ++i) {
      const int32_t donor = all[(size_t)below((int)all.size())];
      int64_t len = 0;
      CHECK(pool.length(donor, &len) == OK);
      const int32_t s = fresh();
      const int how = below(5);
      CHECK(pool.alias(donor, s, 0, how == 0 ? below((int)len + 1) : len) == OK);
      if (how != 1) grow(s, below(how == 2 ? 1000 : 60));
    }
    for (int staged = 0; staged < 2; ++staged) {
      std::vector<int32_t> slots = all, cu = {0};
      std::shuffle(slots.begin(), slots.end(), rng);
      slots.resize((size_t)(1 + below((int)slots.size())));
      for (const int32_t s : slots) {
        int64_t len = 0;
        CHECK(pool.length(s, &len) == OK);
        int delta = below(8) == 0 ? 0 : below(3) ? 1 + below(9) : below(10) ? 1 : 1 + below(400);
        if (!staged) delta = (int)std::min<int64_t>(delta, len);
        cu.push_back(cu.back() + delta);
      }
      check(pool, sh, slots, cu, staged != 0);
    }
  }
  std::printf("ok: shared %lld, pieces %lld, rows stored at once %lld, in arguments %lld, carried %lld\n", (long long)g_shared, (long long)g_pieces,
              (long long)g_direct, (long long)g_inline, (long long)g_carried);
  return 0;
}
