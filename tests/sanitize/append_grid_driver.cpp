// How blocks of an append to the 8-bit cache share its work
// (csrc/jfkv_kv8_append_grid.h): every unit of every head and part is one block's, every
// token's queries are one block's, a unit's blocks are on one XCD where they lie together,
// and places are counted in 32 bits, for the largest sizes as well.  Exits non-zero on the
// first failed check.  Test infrastructure only.
#include <algorithm>
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <random>
#include <vector>

#include "jfkv_kv8_append_grid.h"

using namespace jfkv::kv8::append;

static long g_checks = 0, g_together = 0, g_wide = 0;
#define CHECK(c)                                                                          \
  do {                                                                                    \
    ++g_checks;                                                                           \
    if (!(c)) {                                                                           \
      std::fprintf(stderr, "%s:%d: check failed: %s\n", __FILE__, __LINE__, #c);          \
      std::exit(1);                                                                       \
    }                                                                                     \
  } while (0)

static std::mt19937 g_rng(1);
static int pick(int lo, int hi) { return lo + (int)(g_rng() % (uint32_t)(hi - lo + 1)); }

static void whole_grid(int units, int heads, int parts, int total) {
  const bool together = true;
  std::vector<uint8_t> blocks((size_t)units * heads * parts), tokens(total), plain(total);
  std::vector<int> xcd(units, -1);
  for (int z = 0; z < parts; ++z)
    for (int y = 0; y < heads; ++y)
      for (int x = 0; x < units; ++x) {
        const Place p = place_of(x, y, z, units, heads, parts);
        CHECK(p.unit >= 0 && p.unit < units && p.head >= 0 && p.head < heads && p.part >= 0 && p.part < parts);
        ++blocks[((size_t)p.part * heads + p.head) * units + p.unit];
        const int on = (x + units * (y + heads * z)) % kXcds;
        CHECK(xcd[p.unit] < 0 || xcd[p.unit] == on);
        xcd[p.unit] = on;
      }
  for (uint8_t n : blocks) CHECK(n == 1);
  for (int u = 0; u < units; ++u)
    for (int h = 0; h < heads; ++h) {
      const Tokens a = tokens_of(together, u, units, h, heads, total), b = tokens_of(false, u, units, h, heads, total);
      for (int64_t t = a.first; t < a.end; t += a.step) ++tokens.at(t);
      for (int64_t t = b.first; t < b.end; t += b.step) ++plain.at(t);
    }
  for (int t = 0; t < total; ++t) CHECK(tokens[t] == 1 && plain[t] == 1);
}

int main() {
  for (int turn = 0; turn < 4000; ++turn)
    whole_grid(8 * pick(1, turn % 50 ? 20 : 400), pick(1, turn % 7 ? 9 : 70), pick(2, 3), pick(1, turn % 50 ? 300 : 9000));
  for (int turn = 0; turn < 2000000; ++turn) {
    const int block = 16 << pick(0, 3), rot = 16 * pick(1, 16), parts = pick(2, 3);
    const int heads = turn % 2 ? 1 << pick(0, 15) : pick(1, 65535);
    const int total = (int)(g_rng() >> pick(1, 31)) | 1, B = std::max((int)(g_rng() >> pick(8, 31)), 1);
    // what the entry point lets through
    if ((total / block + 2 * (int64_t)B + 7) * 256 > ((int64_t)1 << 32) - 1) continue;
    const Grid g = grid_of(total, B, block, rot, heads, parts);
    CHECK(g.units >= units_of(total, B, block) && g.units >= 1 && g.units * 256 < (int64_t)1 << 32);
    if (!g.together) continue;
    ++g_together;
    CHECK(g.units % kXcds == 0);
    const int64_t all = g.units * heads * parts;
    g_wide += all > (int64_t)1 << 31;
    // the last block's place, in 32 bits
    CHECK(all <= (int64_t)1 << 32);
    const Place p = place_of(g.units - 1, heads - 1, parts - 1, g.units, heads, parts);
    CHECK(p.unit == g.units - 1 && p.head == heads - 1 && p.part == parts - 1);
  }
  CHECK(g_together > 1000 && g_wide > 10);
  std::printf("%ld checks passed, %ld large grids\n", g_checks, g_together);
  return 0;
}
