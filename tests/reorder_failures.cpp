// The bookkeeping of reordered states where something goes wrong on the way, on the host.  One check a run, by its name.
#include <pthread.h>

#include <atomic>
#include <chrono>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <new>
#include <random>
#include <thread>
#include <vector>

#include "../paper_2605_26289_amd/csrc/pool.hpp"

using namespace dk;

static thread_local long g_fails = -1;  // the allocation that fails, counted from 0 on; < 0: none does
static thread_local bool g_all_fail = false;
static bool take_allocation() { return !g_all_fail && (g_fails < 0 || g_fails-- != 0); }
void* operator new(std::size_t n) {
  void* p = take_allocation() ? std::malloc(n ? n : 1) : nullptr;
  if (!p) throw std::bad_alloc();
  return p;
}
void operator delete(void* p) noexcept { std::free(p); }
void operator delete(void* p, std::size_t) noexcept { std::free(p); }

#define CHECK(x)                                                    \
  do {                                                              \
    if (!(x)) {                                                     \
      std::printf("FAILED line %d: %s (%ld)\n", __LINE__, #x, g_at); \
      std::exit(1);                                                 \
    }                                                               \
  } while (0)
static long g_at = 0;

static int64_t held(Pool& pool) {
  int64_t h = -1;
  pool.stats(&h, nullptr);
  return h;
}
static int32_t slot_of(Pool& pool, int32_t tokens) {
  int32_t s = -1;
  CHECK(pool.acquire(0, 0, &s) == OK);
  const int32_t cu[2] = {0, tokens};
  CHECK(pool.append(1, &s, cu, nullptr, nullptr) == OK);
  return s;
}

// A node that cannot grow takes no granule from the allocator, and no run of free ones is forgotten.
static void granules() {
  long failures = 0;
  for (int gap = 0; gap < 4; ++gap) {
    for (g_at = 0;; ++g_at) {
      GranuleAllocator alloc(32);
      for (int g = 0; g < 32; g += 1 + gap) CHECK(alloc.take(g));  // (gaps of 0 .. 3)
      if (gap == 0) alloc.give_back(3), alloc.give_back(4), alloc.give_back(9);
      const int64_t free0 = alloc.free_count();
      bool thrown = false;
      {
        Node n(&alloc, 16, nullptr, 0);
        g_fails = g_at;
        try {
          n.grow(16 * 3 - 5);
        } catch (const std::bad_alloc&) {
          thrown = true;
        }
        g_fails = -1;
        CHECK(alloc.free_count() == free0 - (int64_t)n.granules.size());
        if (thrown) CHECK(n.len == 0);
      }
      CHECK(alloc.free_count() == free0);
      int64_t found = 0;
      while (alloc.take_first() >= 0) ++found;
      CHECK(found == free0);
      if (!thrown) break;
      ++failures;
    }
  }
  for (g_at = 0; g_at < 3; ++g_at) {  // out of the middle of a run, off its ends
    const int64_t which[3] = {5, 0, 15};
    GranuleAllocator alloc(16);
    bool taken = false;
    g_fails = 0;
    try {
      taken = alloc.take(which[g_at]);
    } catch (const std::bad_alloc&) {
      ++failures;
    }
    g_fails = -1;
    CHECK(alloc.free_count() == (taken ? 15 : 16));
    int64_t found = 0;
    while (alloc.take_first() >= 0) ++found;
    CHECK(found == (taken ? 15 : 16));
  }
  CHECK(failures > 4);
}

// Giving cells back needs no memory: it is done where sequences end, in destructors too.
static void giving_back() {
  for (g_at = 0; g_at < 40; ++g_at) {
    std::mt19937 rng((unsigned)g_at);
    const int n = 1 + (int)(rng() % 70);
    GranuleAllocator alloc(n);
    std::vector<int64_t> taken;
    taken.reserve((size_t)n);
    std::vector<char> free_now((size_t)n, 1);
    for (int turn = 0; turn < 300; ++turn) {
      const int what = (int)(rng() % 4);
      const int64_t some = (int64_t)(rng() % (unsigned)n);
      const int64_t g = what == 0 ? alloc.take_first() : what == 1 ? alloc.take_fresh() : alloc.take(some) ? some : -1;
      if (what < 2) CHECK((g >= 0) == ((int64_t)taken.size() < n));
      if (g >= 0) {
        CHECK(free_now[(size_t)g]);
        free_now[(size_t)g] = 0;
        taken.push_back(g);
      }
      g_all_fail = true;
      if (turn % 60 > 40) {
        const size_t back = (size_t)(rng() % (unsigned)(taken.size() + 1));
        for (size_t i = 0; i < back; ++i) {
          const size_t k = (size_t)(rng() % (unsigned)taken.size());
          alloc.give_back(taken[k]);
          free_now[(size_t)taken[k]] = 1;
          taken[k] = taken.back();
          taken.pop_back();
        }
      }
      g_all_fail = false;
      CHECK(alloc.free_count() == n - (int64_t)taken.size());
    }
    for (int64_t g = 0; g < n; ++g)
      if (free_now[(size_t)g]) CHECK(alloc.take_first() == g);
    CHECK(alloc.take_first() == -1 && alloc.free_count() == 0);
  }
}

// Whichever allocation of the call fails: every slot is what it was, and nothing refers to its cells but itself.
static void out_of_memory() {
  long failures = 0;
  for (g_at = 0;; ++g_at) {
    Pool pool(8, 0, 64 * 16, 16);
    std::vector<int32_t> slots;
    for (int i = 0; i < 6; ++i) slots.push_back(slot_of(pool, 40 + 3 * i));
    std::vector<std::vector<int64_t>> before;
    for (int32_t s : slots) {
      before.emplace_back(64, -1);
      CHECK(pool.cells(s, before.back().data(), 64) == OK);
    }
    const std::vector<int32_t> parents = {0, 0, 0, 3, 3, 1};
    const int64_t full = held(pool);
    Pool::Reorder re;
    bool thrown = false;
    g_fails = g_at;
    try {
      (void)pool.reorder(6, slots.data(), parents.data(), &re);
    } catch (const std::bad_alloc&) {
      thrown = true;
    }
    g_fails = -1;
    if (!thrown) {
      pool.settle_reorder(&re);
      break;
    }
    ++failures;
    CHECK(held(pool) == full);
    for (size_t i = 0; i < slots.size(); ++i) {
      int64_t len = 0;
      CHECK(pool.length(slots[i], &len) == OK && len == 40 + 3 * (int64_t)i);
      std::vector<int64_t> now(64, -1);
      CHECK(pool.cells(slots[i], now.data(), 64) == OK && now == before[i]);
    }
    // nothing shares them: cells come back as soon as they are trimmed, all of them when the slots go
    CHECK(pool.trim(slots[0], 8) == OK);
    CHECK(held(pool) == full - 2 * 16);
    for (int32_t s : slots) CHECK(pool.release(s) == OK);
    CHECK(held(pool) == 0);
  }
  CHECK(failures > 10);
}

// Between a reorder and its end (kept or taken back) no other thread's call comes in: what is taken back is what was there.
static void one_step() {
  for (g_at = 0; g_at < 2; ++g_at) {
    Pool pool(8, 0, 64 * 16, 16);
    std::vector<int32_t> slots;
    for (int i = 0; i < 4; ++i) slots.push_back(slot_of(pool, 40 + 3 * i));
    const std::vector<int32_t> parents = {0, 0, 0, 0};
    Pool::Reorder re;
    CHECK(pool.reorder(4, slots.data(), parents.data(), &re) == OK);
    std::atomic<bool> started{false};
    int32_t released = -1, acquired = -1, fresh = -1;
    std::thread other([&] {
      started = true;
      released = pool.release(slots[2]);
      acquired = pool.acquire(0, 0, &fresh);
    });
    while (!started) std::this_thread::yield();
    std::this_thread::sleep_for(std::chrono::milliseconds(100));  // (a call that could come in has, by now)
    if (g_at == 0) pool.undo_reorder(4, slots.data(), &re);
    else pool.settle_reorder(&re);
    other.join();
    CHECK(released == OK && acquired == OK);
    for (int i = 0; i < 4; ++i) {
      int64_t len = -1;
      const int32_t rc = pool.length(slots[(size_t)i], &len);
      if (i == 2 && fresh != slots[2]) CHECK(rc == ERR_NO_SLOT);
      else CHECK(rc == OK && len == (i == 2 ? 0 : g_at == 0 ? 40 + 3 * i : 40));
    }
    int64_t len = -1;
    CHECK(pool.length(fresh, &len) == OK && len == 0);
    for (int i = 0; i < 4; ++i)
      if (i != 2) CHECK(pool.release(slots[(size_t)i]) == OK);
    CHECK(held(pool) == 0);
  }
}

// Searches on threads of their own, some of their calls taken back, while others acquire, alias, trim and release.
static void threads() {
  constexpr int kThreads = 5, kSteps = 1500;
  Pool pool(4 * kThreads + 1, 0, 1 << 14, 16);
  const int32_t prompt = slot_of(pool, 100);
  std::atomic<int> failures{0};
  const auto search = [&](int id) {
    std::mt19937 rng(500 + (unsigned)id);
    Pool::Reorder re;
    std::vector<int32_t> slots;
    std::vector<int64_t> lens;
    for (int step = 0; step < kSteps; ++step) {
      if (slots.empty()) {
        for (int i = 0; i < 4; ++i) {
          int32_t s = -1;
          if (pool.acquire(0, -1, &s) != OK || pool.alias(prompt, s, 0, 90 + i) != OK) ++failures;
          slots.push_back(s);
          lens.push_back(90 + i);
        }
      }
      std::vector<int32_t> parents, cu = {0};
      for (int i = 0; i < 4; ++i) {
        parents.push_back((int32_t)(rng() % 4));
        cu.push_back(i + 1);
      }
      const int32_t rc = pool.reorder(4, slots.data(), parents.data(), &re);
      if (rc == OK && rng() % 3 == 0) {
        pool.undo_reorder(4, slots.data(), &re);
      } else if (rc == OK) {
        pool.settle_reorder(&re);
        std::vector<int64_t> after;
        for (int i = 0; i < 4; ++i) after.push_back(lens[(size_t)parents[(size_t)i]]);
        lens = after;
      } else if (rc != ERR_NO_CELLS) {
        ++failures;
      }
      if (pool.append(4, slots.data(), cu.data(), nullptr, nullptr) == OK)
        for (int64_t& l : lens) ++l;
      if (rng() % 8 == 0) {
        const size_t i = rng() % 4;
        lens[i] -= (int64_t)(rng() % 5);
        if (pool.trim(slots[i], lens[i]) != OK) ++failures;
      }
      for (int i = 0; i < 4; ++i) {
        int64_t len = -1;
        if (pool.length(slots[(size_t)i], &len) != OK || len != lens[(size_t)i]) ++failures;
      }
      if (step % 60 == 59) {
        for (int32_t s : slots)
          if (pool.release(s) != OK) ++failures;
        slots.clear();
        lens.clear();
      }
    }
    for (int32_t s : slots)
      if (pool.release(s) != OK) ++failures;
  };
  std::vector<std::thread> all;
  for (int i = 0; i < kThreads; ++i) all.emplace_back(search, i);
  for (std::thread& t : all) t.join();
  CHECK(failures == 0);
  CHECK(pool.release(prompt) == OK);
  CHECK(held(pool) == 0);
}

// Cells that no slot sees any more are free after the call, but for what is left of a granule.
static int32_t alias_of(Pool& pool, int32_t donor, int64_t n) {
  int32_t s = -1;
  CHECK(pool.acquire(0, 0, &s) == OK && pool.alias(donor, s, 0, n) == OK);
  return s;
}
static int32_t append_to(Pool& pool, int32_t s, int32_t n) {
  const int32_t cu[2] = {0, n};
  return pool.append(1, &s, cu, nullptr, nullptr);
}
static int32_t reorder(Pool& pool, const std::vector<int32_t>& slots, const std::vector<int32_t>& parents) {
  Pool::Reorder re;
  const int32_t rc = pool.reorder((int32_t)slots.size(), slots.data(), parents.data(), &re);
  if (rc == OK) pool.settle_reorder(&re);
  return rc;
}
static void cells_come_back() {
  {  // a long state goes, its beginning is another's prefix
    Pool pool(4, 0, 2048, 256);
    const int32_t a = slot_of(pool, 64), b = alias_of(pool, a, 64);
    CHECK(append_to(pool, a, 1500) == OK && held(pool) == 7 * 256);
    CHECK(reorder(pool, {a, b}, {1, 1}) == OK && held(pool) == 256);
    CHECK(append_to(pool, b, 600) == OK);
    int64_t len = 0;
    CHECK(pool.length(a, &len) == OK && len == 64);
  }
  {  // cells of a sequence that is gone, seen by a state that goes now, through a node of its own without a token
    Pool pool(8, 0, 4096, 256);
    const int32_t p = slot_of(pool, 1500), a = alias_of(pool, p, 1400), b = alias_of(pool, p, 64);
    CHECK(pool.release(p) == OK && held(pool) >= 6 * 256);
    CHECK(reorder(pool, {a, b}, {1, 1}) == OK && held(pool) == 256);
  }
  {  // the child that saw most goes later, in another call; one that sees as much stays
    Pool pool(8, 0, 8192, 256);
    const int32_t a = slot_of(pool, 64);
    CHECK(append_to(pool, a, 1936) == OK);  // eight granules
    const int32_t b = alias_of(pool, a, 1900), c = alias_of(pool, a, 1900), d = alias_of(pool, a, 300), e = slot_of(pool, 3);
    CHECK(reorder(pool, {a, e}, {1, 1}) == OK && held(pool) == 8 * 256 + 2 * 256);
    CHECK(reorder(pool, {b, e}, {1, 1}) == OK && held(pool) == 8 * 256 + 3 * 256);
    CHECK(reorder(pool, {c, d}, {1, 1}) == OK && held(pool) == 2 * 256 + 3 * 256);
    CHECK(append_to(pool, c, 5) == OK && append_to(pool, d, 5) == OK);
    int64_t len = 0;
    CHECK(pool.length(c, &len) == OK && len == 305);
    std::vector<int64_t> x(305), y(305);
    CHECK(pool.cells(c, x.data(), 305) == OK && pool.cells(d, y.data(), 305) == OK);
    for (int i = 0; i < 305; ++i) CHECK((x[(size_t)i] == y[(size_t)i]) == (i < 300));
  }
  {  // a state that goes in the same call in which another slot takes it over stays whole, and so does one that is taken back
    Pool pool(8, 0, 8192, 256);
    const int32_t a = slot_of(pool, 1000), b = alias_of(pool, a, 100), c = slot_of(pool, 7);
    CHECK(reorder(pool, {a, b, c}, {2, 1, 0}) == OK);
    int64_t len = 0;
    CHECK(pool.length(c, &len) == OK && len == 1000 && held(pool) == 4 * 256 + 256);
    std::vector<int32_t> slots = {a, b, c}, parents = {1, 1, 1};
    Pool::Reorder re;
    CHECK(pool.reorder(3, slots.data(), parents.data(), &re) == OK);
    pool.undo_reorder(3, slots.data(), &re);
    CHECK(pool.length(c, &len) == OK && len == 1000 && held(pool) == 5 * 256);
    std::vector<int64_t> x(1000);
    CHECK(pool.cells(c, x.data(), 1000) == OK);
    std::vector<char> seen(8192, 0);
    for (int64_t cell : x) CHECK(cell >= 0 && !seen[(size_t)cell]++);
    CHECK(append_to(pool, c, 24) == OK && held(pool) == 5 * 256);
  }
  // a search that goes on: what is held stays within some granules of what the slots see
  for (int beams : {2, 5, 16}) {
    g_at = beams;
    Pool pool(40, 0, 256 * 4096, 256);
    std::mt19937 rng((unsigned)beams);
    const int32_t prompt = slot_of(pool, 1000);
    std::vector<int32_t> slots, cu = {0};
    for (int i = 0; i < beams; ++i) {
      slots.push_back(alias_of(pool, prompt, 1000));
      cu.push_back(i + 1);
    }
    CHECK(pool.release(prompt) == OK);
    for (int step = 0; step < 3000; ++step) {
      std::vector<int32_t> parents;
      for (int i = 0; i < beams; ++i) parents.push_back((int32_t)(rng() % (unsigned)beams));
      CHECK(reorder(pool, slots, parents) == OK && pool.append(beams, slots.data(), cu.data(), nullptr, nullptr) == OK);
      if (step % 100 != 99) continue;
      std::vector<char> granule(4096, 0);
      int64_t granules = 0;
      for (int32_t s : slots) {
        int64_t len = 0;
        CHECK(pool.length(s, &len) == OK && len == 1001 + step);
        std::vector<int64_t> x((size_t)len);
        CHECK(pool.cells(s, x.data(), len) == OK);
        for (int64_t cell : x) {
          granules += granule[(size_t)(cell / 256)] == 0;
          granule[(size_t)(cell / 256)] = 1;
        }
      }
      CHECK(held(pool) == 256 * granules);  // no granule without a cell that some slot sees
    }
    for (int32_t s : slots) CHECK(pool.release(s) == OK);
    CHECK(held(pool) == 0);
  }
}

// A search's chain of nodes is as long as the search: letting go of it does not need a stack as deep.
static void long_chains() {
  const int steps = 20000;
  Pool pool(2, 0, 2 * steps + 64, 1);
  const std::vector<int32_t> slots = {slot_of(pool, 1), slot_of(pool, 1)}, cu = {0, 1, 2};
  for (int step = 0; step < steps; ++step) {
    const int32_t parent = step & 1;
    CHECK(reorder(pool, slots, {parent, parent}) == OK);
    CHECK(pool.append(2, slots.data(), cu.data(), nullptr, nullptr) == OK);
  }
  int64_t runs = 0, depth = 0, len = 0;
  CHECK(pool.seq_stats(slots[0], &runs, &depth) == OK && depth > steps / 2);
  CHECK(pool.length(slots[0], &len) == OK && len == steps + 1);
  pthread_attr_t small;
  pthread_attr_init(&small);
  pthread_attr_setstacksize(&small, 512 << 10);
  struct Both {
    Pool* pool;
    const std::vector<int32_t>* slots;
  } both{&pool, &slots};
  pthread_t t;
  CHECK(pthread_create(&t, &small, [](void* p) -> void* {
    const Both& b = *(const Both*)p;
    for (int32_t s : *b.slots) CHECK(b.pool->release(s) == OK);
    return nullptr;
  }, &both) == 0);
  pthread_join(t, nullptr);
  CHECK(held(pool) == 0);
}

int main(int argc, char** argv) {
  const char* what = argc > 1 ? argv[1] : "";
  if (!std::strcmp(what, "granules")) granules();
  else if (!std::strcmp(what, "giving_back")) giving_back();
  else if (!std::strcmp(what, "out_of_memory")) out_of_memory();
  else if (!std::strcmp(what, "one_step")) one_step();
  else if (!std::strcmp(what, "cells_come_back")) cells_come_back();
  else if (!std::strcmp(what, "long_chains")) long_chains();
  else if (!std::strcmp(what, "threads")) threads();
  else return 2;
  std::printf("ok\n");
  return 0;
}
