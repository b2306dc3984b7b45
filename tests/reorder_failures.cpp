// The bookkeeping of reordered states where something goes wrong on the way, on the host.  One check a run, by its name.
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <new>
#include <vector>

#include "../paper_2605_26289_amd/csrc/pool.hpp"

using namespace dk;

static long g_fails = -1;  // the allocation that fails, counted from 0 on; < 0: none does
static bool take_allocation() { return g_fails < 0 || g_fails-- != 0; }
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

int main(int argc, char** argv) {
  const char* what = argc > 1 ? argv[1] : "";
  if (!std::strcmp(what, "granules")) granules();
  else return 2;
  std::printf("ok\n");
  return 0;
}
