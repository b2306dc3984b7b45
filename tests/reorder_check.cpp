// Pool::reorder against a model, on the host: cells hold numbers, moves copy them, and after every operation every sequence reads what
// the model says.  Small granules, aliases, trims, releases, borrowed tails, states taken back.
#include <algorithm>
#include <cstdio>
#include <cstdlib>
#include <random>
#include <vector>

#include "../paper_2605_26289_amd/csrc/pool.hpp"

using namespace dk;

static int g_seed = 0, g_turn = 0;
#define CHECK(x)                                                                          \
  do {                                                                                    \
    if (!(x)) {                                                                           \
      std::printf("FAILED line %d: %s (seed %d, turn %d)\n", __LINE__, #x, g_seed, g_turn); \
      std::exit(1);                                                                       \
    }                                                                                     \
  } while (0)

int main(int argc, char** argv) {
  const int seeds = argc > 1 ? std::atoi(argv[1]) : 200;
  long long moved = 0, aliased = 0, refused = 0;
  for (int seed = 0; seed < seeds; ++seed) {
    g_seed = seed;
    std::mt19937 rng(seed);
    const auto below = [&](int n) { return (int)(rng() % (unsigned)std::max(1, n)); };
    const int granule = seed % 10 == 9 ? 256 : 1 + below(16), cells = granule * (seed % 4 == 0 ? 40 : 400), kSlots = 12;
    Pool pool(kSlots, 0, cells, granule);
    std::vector<int> memory((size_t)cells, -1);
    std::vector<std::vector<int>> model(kSlots);
    std::vector<char> used(kSlots, 0);
    int next = 0;
    Pool::Reorder re;
    const auto verify = [&]() {
      for (int s = 0; s < kSlots; ++s) {
        if (!used[(size_t)s]) continue;
        int64_t len = 0;
        CHECK(pool.length(s, &len) == OK && len == (int64_t)model[(size_t)s].size());
        std::vector<int64_t> c((size_t)len);
        CHECK(pool.cells(s, c.data(), len) == OK);
        for (int64_t i = 0; i < len; ++i) CHECK(memory[(size_t)c[(size_t)i]] == model[(size_t)s][(size_t)i]);
      }
    };
    for (g_turn = 0; g_turn < 300; ++g_turn) {
      std::vector<int32_t> live;
      for (int s = 0; s < kSlots; ++s)
        if (used[(size_t)s]) live.push_back(s);
      const int what = below(10);
      if (live.size() < 3 || (what == 0 && live.size() < (size_t)kSlots)) {
        int32_t s = -1;
        CHECK(pool.acquire(0, 0, &s) == OK);
        used[(size_t)s] = 1;
        model[(size_t)s].clear();
        if (!live.empty() && below(3)) {
          const int32_t donor = live[(size_t)below((int)live.size())];
          const int m = below(3) ? (int)model[(size_t)donor].size() : below((int)model[(size_t)donor].size() + 1);
          CHECK(pool.alias(donor, s, 0, m) == OK);
          model[(size_t)s].assign(model[(size_t)donor].begin(), model[(size_t)donor].begin() + m);
        }
      } else if (what <= 3) {
        const int32_t s = live[(size_t)below((int)live.size())];
        const int32_t cu[2] = {0, below(4) ? 1 : below(3 * granule + 2)};
        std::vector<int64_t> dst;
        const int32_t rc = pool.append(1, &s, cu, nullptr, &dst);
        CHECK(rc == OK || rc == ERR_NO_CELLS);
        if (rc == OK)
          for (const int64_t c : dst) {
            memory[(size_t)c] = next;
            model[(size_t)s].push_back(next++);
          }
      } else if (what == 4) {
        const int32_t s = live[(size_t)below((int)live.size())];
        const int to = below(2) ? std::max(0, (int)model[(size_t)s].size() - 1) : below((int)model[(size_t)s].size() + 1);
        CHECK(pool.trim(s, to) == OK);
        model[(size_t)s].resize((size_t)to);
      } else if (what == 5 && below(3) == 0) {
        const int32_t s = live[(size_t)below((int)live.size())];
        CHECK(pool.release(s) == OK);
        used[(size_t)s] = 0;
      } else {
        std::shuffle(live.begin(), live.end(), rng);
        live.resize((size_t)(1 + below((int)live.size())));
        std::vector<int32_t> parents;
        for (size_t i = 0; i < live.size(); ++i) parents.push_back(below((int)live.size()));
        std::vector<std::vector<int>> after;
        for (size_t i = 0; i < live.size(); ++i) after.push_back(model[(size_t)live[(size_t)parents[i]]]);
        int64_t held0 = 0, held1 = 0, free0 = 0;
        pool.stats(&held0, &free0);
        const int32_t rc = pool.reorder((int32_t)live.size(), live.data(), parents.data(), &re);
        CHECK(rc == OK || rc == ERR_NO_CELLS);
        if (rc == ERR_NO_CELLS) {
          ++refused;
        } else if (below(5) == 0) {  // a launch that failed
          pool.undo_reorder((int32_t)live.size(), live.data(), &re);
          pool.stats(&held1, nullptr);
          CHECK(held1 == held0);
        } else {
          for (const Pool::Move& m : re.moves) {
            CHECK(m.len > 0 && m.len < (granule == 256 ? 256 : granule));
            for (int64_t i = 0; i < m.len; ++i) {
              CHECK(m.to + i < m.from || m.to + i >= m.from + m.len);
              memory[(size_t)(m.to + i)] = memory[(size_t)(m.from + i)];
            }
            ++moved;
          }
          aliased += (long long)(live.size() - re.moves.size());
          pool.settle_reorder(&re);
          for (size_t i = 0; i < live.size(); ++i) model[(size_t)live[i]] = after[i];
        }
      }
      verify();
    }
    for (int s = 0; s < kSlots; ++s)
      if (used[(size_t)s]) CHECK(pool.release(s) == OK);
    int64_t held = -1, left = 0;
    pool.stats(&held, &left);
    CHECK(held == 0 && left == cells);
    // what a beam search does: chains stay short however long it goes on
    std::vector<int32_t> beams;
    int32_t prompt = -1;
    CHECK(pool.acquire(0, 0, &prompt) == OK);
    const int32_t pc[2] = {0, granule + 1};
    CHECK(pool.append(1, &prompt, pc, nullptr, nullptr) == OK);
    for (int b = 0; b < 4; ++b) {
      int32_t s = -1;
      CHECK(pool.acquire(0, 0, &s) == OK && pool.alias(prompt, s, 0, granule + 1) == OK);
      beams.push_back(s);
    }
    const int unit = granule == 256 ? 64 : granule, steps = granule == 256 ? 600 : std::min(60, 6 * granule);
    for (int step = 0; step < steps; ++step) {
      std::vector<int32_t> parents, cu = {0};
      for (int b = 0; b < 4; ++b) {
        parents.push_back(below(4));
        cu.push_back(b + 1);
      }
      CHECK(pool.reorder(4, beams.data(), parents.data(), &re) == OK);
      pool.settle_reorder(&re);
      CHECK(pool.append(4, beams.data(), cu.data(), nullptr, nullptr) == OK);
      for (int b = 0; b < 4; ++b) {
        int64_t segs = 0, depth = 0, len = 0;
        CHECK(pool.seq_stats(beams[(size_t)b], &segs, &depth) == OK && pool.length(beams[(size_t)b], &len) == OK);
        CHECK(len == granule + 2 + step && depth <= 3 + (step + 1) / unit && segs <= 4 + (step + 1) / unit);
      }
    }
  }
  std::printf("ok: copied %lld, taken over or aliased %lld, refused %lld\n", moved, aliased, refused);
  return 0;
}
