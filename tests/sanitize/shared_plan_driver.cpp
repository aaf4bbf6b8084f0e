// Carries out the plan of the attention of requests that share prefixes
// (csrc/jfkv_kv8_shared_plan.h) for many batches, as the kernels' blocks do, and checks
// that every step of every unit is in exactly one segment, that every record that the
// join reads has been written, and by nobody else, and that all of them lie in the
// workspace.  Under AddressSanitizer and UndefinedBehaviorSanitizer.  Exits non-zero on
// the first failed check.  Test infrastructure only.
#include <algorithm>
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <random>
#include <vector>

#include "jfkv_kv8_shared_plan.h"

using namespace jfkv::kv8::shared;

static long g_checks = 0, g_lines = 0, g_shares = 0, g_tight = 0;
static const char* g_name = "";
#define CHECK(c)                                                                          \
  do {                                                                                    \
    ++g_checks;                                                                           \
    if (!(c)) {                                                                           \
      std::fprintf(stderr, "%s:%d: check failed: %s (%s)\n", __FILE__, __LINE__, #c, g_name); \
      std::exit(1);                                                                       \
    }                                                                                     \
  } while (0)

static std::mt19937 g_rng(1);
static int pick(int lo, int hi) { return lo + (int)(g_rng() % (uint32_t)(hi - lo + 1)); }

// A call's sizes, groups and lengths.
struct Call {
  int B, G, sq, Hkv, gq, own_kind, group_gap, own_gap, own_info, own_recs;
};
struct Batch {
  std::vector<int> bounds, most, lens;
  bool valid = true;
  int first(int g) const { return bounds[g]; }
  int length(int b) const { return lens[b]; }
  int of(int b) const {
    return (int)(std::upper_bound(bounds.begin(), bounds.end() - 1, b) - bounds.begin()) - 1;
  }
  int shared(int g) const {
    if (!valid || first(g + 1) - first(g) < 2) return 0;
    return std::min(std::max(most[g], 0), length(first(g)));
  }
};
static Batch batch_of(const std::vector<int>& sizes, const std::vector<int>& most, const std::vector<int>& lens) {
  Batch b;
  b.bounds = {0};
  for (int n : sizes) b.bounds.push_back(b.bounds.back() + n);
  b.most = most, b.lens = lens;
  CHECK((size_t)b.bounds.back() == lens.size() && sizes.size() == most.size());
  return b;
}

struct Record {
  int64_t from;  // columns
  int cols;
};
// What the blocks of all kernels leave.
struct Left {
  std::vector<int> block, records, col, cols;  // of each entry of `info` (block -1: none)
  std::vector<Record> written;
};

template <int D, int PART>
static void kernel(const Call& a, const Batch& batch, int blocks, int threads, Left& left) {
  const int teams = threads / 64, n = items_of<PART>(a);
  std::vector<Item> items(n);
  std::vector<int64_t> upto(n + 1, 0);
  std::vector<std::vector<std::vector<int>>> blocks_of(n);  // of each unit's segments
  std::vector<std::vector<std::vector<int>>> seen(n);       // how often each of its steps
  int64_t work = 0, begins = 0;
  int count = 0;
  for (int i = 0; i < n; ++i) {
    const Item t = items[i] = item_of<D, PART>(a, batch, i);
    const int m = t.work() ? t.chunks() * a.Hkv : 0;
    work += t.work() * m, count += m, begins += (int64_t)m * start_of(t.kind);
    upto[i + 1] = upto[i] + t.span() * m;
    blocks_of[i].resize(m);
    seen[i].assign(m, std::vector<int>(t.steps(), 0));
    CHECK(t.kind == kRows1 || t.kind == kRows2 || PART == kGroups);
    CHECK(t.work() == 0 || (t.lo >= 0 && t.hi <= batch.length(t.request)));
  }
  CHECK(upto[n] == work + begins);
  if (count == 0) return;

  const auto put = [&](int block, int i, const Cut& c) {
    const Item& t = items[i];
    const Spot s = spot_of(a, t, c.u);
    const bool own = PART == kOwn || (PART == kBoth && i >= 2 * a.G);
    const int cols = std::min(width_of(t.kind), t.cols - s.col), entry = own ? a.own_info + s.at : s.at;
    CHECK(c.u >= 0 && c.u < (int)seen[i].size() && s.kv >= 0 && s.kv < a.Hkv && s.col < t.cols && cols > 0);
    CHECK(c.r0 >= 0 && c.r1 <= t.steps());
    if (c.r0 == 0 && c.r1 > 0) {
      CHECK(left.block.at(entry) < 0);
      left.block[entry] = block, left.records[entry] = c.records;
      left.col[entry] = t.request * a.gq * a.sq + s.col, left.cols[entry] = cols;
    }
    if (c.r0 >= c.r1) return false;
    for (int r = c.r0; r < c.r1; ++r) ++seen[i][c.u][r];
    blocks_of[i][c.u].push_back(block);
    left.written.push_back({record_of(a, own, block, s.at), cols});
    CHECK(left.written.back().from >= (own ? a.own_recs : 0));
    CHECK(own || left.written.back().from + cols <= a.own_recs);
    return true;
  };
  if (takes_line(work, count, blocks, n, threads)) {
    ++g_lines;
    const int64_t piece = piece_of<D, PART>(work + begins, blocks);
    CHECK(piece * blocks >= work + begins);
    for (const Item& t : items) CHECK(t.work() == 0 || cost_of(t.kind) <= piece);
    g_tight += piece < 40;
    for (int block = 0; block < blocks; ++block) {
      const int64_t begin = block * piece, end = std::min(begin + piece, work + begins);
      for (int64_t x = begin; x < end;) {
        const int i = (int)(std::upper_bound(upto.begin(), upto.end(), x) - upto.begin()) - 1;
        const Cut c = cut_line(items[i], upto[i], x, begin, end, piece);
        CHECK(c.next > x);
        put(block, i, c);
        x = c.next;
      }
    }
  } else {
    ++g_shares;
    CHECK(n <= threads);
    float most = 0.0f;
    for (int team = teams - 1; team >= 0; --team) {
      const float length = share_length(work, count, blocks, team, teams);
      int many = 0;
      for (int i = 0; i < n; ++i)
        if (items[i].work()) many += shares((int)items[i].work(), length) * (items[i].chunks() * a.Hkv);
      if (team == teams - 1) CHECK(many <= blocks);
      if (team == teams - 1 || many <= blocks) most = length;
    }
    int block = 0;
    for (int i = 0; i < n; ++i) {
      const int each = shares((int)items[i].work(), most), all = each * (int)seen[i].size();
      for (int j = 0; j < all; ++j) put(block++, i, cut_share(items[i], each, j));
    }
    CHECK(block <= blocks);
  }
  for (int i = 0; i < n; ++i)
    for (size_t u = 0; u < seen[i].size(); ++u) {
      for (int times : seen[i][u]) CHECK(times == 1);
      const Spot s = spot_of(a, items[i], (int)u);
      const bool own = PART == kOwn || (PART == kBoth && i >= 2 * a.G);
      const int entry = own ? a.own_info + s.at : s.at;
      CHECK(left.block.at(entry) >= 0);
      // the records that are counted are those that have been written
      CHECK(left.records[entry] == (int)blocks_of[i][u].size());
      for (size_t k = 0; k < blocks_of[i][u].size(); ++k)
        CHECK(blocks_of[i][u][k] == left.block[entry] + (int)k);
    }
}

template <int D>
static void call(const Batch& batch, int Hkv, int gq, int sq, bool both, int cus, const char* name) {
  g_name = name;
  const int B = (int)batch.lens.size(), G = (int)batch.most.size(), pairs = gq * sq, columns = B * Hkv * pairs;
  CHECK(columns <= 65536);
  jf_kv_layout L = {};
  L.head_dim = D, L.num_kv_heads = Hkv;
  const Layout p = layout_of(L, B, sq, Hkv * gq, both, cus);
  const Call a = {B, G, sq, Hkv, gq, p.own_kind, p.group_gap, p.own_gap, p.own_info, p.own_recs};
  Left left;
  left.block.assign(2 * columns, -1), left.records.assign(2 * columns, 0);
  left.col = left.cols = left.records;
  if (both) {
    kernel<D, kBoth>(a, batch, p.own_blocks, 64 * kRowWaves, left);
  } else {
    kernel<D, kGroups>(a, batch, p.group_blocks, 512, left);
    kernel<D, kOwn>(a, batch, p.own_blocks, 64 * kRowWaves, left);
  }
  // all records apart, and in the workspace
  std::sort(left.written.begin(), left.written.end(), [](Record x, Record y) { return x.from < y.from; });
  int64_t end = 0;
  for (const Record& r : left.written) {
    CHECK(r.from >= end);
    end = r.from + r.cols;
  }
  CHECK(p.recs >= sizeof(int2) * 2 * (size_t)columns && p.recs % 16 == 0);
  CHECK(p.recs + (size_t)end * (D + 4) * sizeof(float) <= p.bytes);
  // the join finds the chunk of every column
  const int step = std::max(1, B / 300);
  for (int b = 0; b < B; b += step) {
    const int g = batch.valid ? batch.of(b) : 0, shared = batch.shared(g);
    for (int kv = 0; kv < Hkv; kv += std::max(1, Hkv - 1))
      for (int pair = 0; pair < pairs; ++pair) {
        const int column = b * pairs + pair;
        if (shared > 0) {
          const Asked ask = group_of<D>(a, both, batch.first(g), batch.first(g + 1), b, pair, kv);
          CHECK(left.block.at(ask.at) >= 0 && left.col[ask.at] + ask.in == column);
          CHECK(ask.in >= 0 && ask.in < left.cols[ask.at]);
        }
        if (batch.length(b) > shared) {
          const Asked ask = own_of(a, b, pair, kv);
          const int entry = a.own_info + ask.at;
          CHECK(left.block.at(entry) >= 0 && left.col[entry] + ask.in == column);
          CHECK(ask.in >= 0 && ask.in < left.cols[entry]);
        }
      }
  }
}
static void calls(const Batch& batch, int Hkv, int gq, int sq, int D, int cus, const char* name) {
  for (bool both : {false, true}) {
    if (D == 64) call<64>(batch, Hkv, gq, sq, both, cus, name);
    if (D == 128) call<128>(batch, Hkv, gq, sq, both, cus, name);
    if (D == 256) call<256>(batch, Hkv, gq, sq, both, cus, name);
  }
}

// `alone` requests by themselves, then groups of `size` that share `most` positions.
static Batch mixed(int alone, int groups, int size, int most, int own) {
  std::vector<int> sizes(alone, 1), shared(alone, 0), lens(alone, own);
  for (int g = 0; g < groups; ++g) {
    sizes.push_back(size), shared.push_back(most);
    lens.insert(lens.end(), size, most + own);
  }
  return batch_of(sizes, shared, lens);
}
static Batch with_pairs(int pairs, int most, int size, int more) {
  Batch b = mixed(0, pairs, 2, most, 5);
  b.bounds.push_back(b.bounds.back() + size);
  b.most.push_back(more);
  b.lens.insert(b.lens.end(), size, more + 5);
  return b;
}

static Batch any_batch(int room) {  // of at most `room` requests
  std::vector<int> sizes, shared, lens;
  const int kinds = pick(0, 5), longest = 1 << pick(0, 14);
  const int wanted = std::min(room, pick(0, 3) ? pick(1, 80) : pick(1, 1500));
  while ((int)lens.size() < wanted) {
    int n = kinds == 0 ? 1 : kinds == 1 ? pick(1, 3) : kinds == 2 ? pick(0, 40) : kinds == 3 ? pick(30, 300)
            : pick(0, 9) ? 1 : pick(20, 120);
    n = std::min(n, wanted - (int)lens.size());
    const int most = pick(0, 4) ? pick(0, longest) : 0;
    sizes.push_back(n), shared.push_back(most);
    for (int i = 0; i < n; ++i)
      lens.push_back(pick(0, 12) ? pick(0, 1) * most + pick(0, std::max(1, longest / 8)) : 0);
  }
  if (sizes.size() > lens.size()) sizes.clear();  // (more groups than requests: refused)
  return sizes.empty() ? mixed(1, 0, 0, 0, 1) : batch_of(sizes, shared, lens);
}

int main() {
  // pieces that are shorter than a step of the widest tiles
  for (int D : {64, 128, 256}) {
    calls(mixed(300, 1, 64, 512, 30), 8, 4, 1, D, 256, "300 alone, 64 that share 512");
    calls(mixed(256, 1, 64, 1024, 9), 8, 4, 1, D, 256, "256 alone, 64 that share 1,024");
    calls(with_pairs(17, 32, 64, 128), 8, 4, 1, D, 256, "17 pairs, 64 that share 128");
    calls(with_pairs(16, 32, 64, 320), 8, 4, 1, D, 256, "16 pairs, 64 that share 320");
    for (int most = 65; most <= 4096; most += 311)
      for (int alone : {257, 311, 420})
        for (int size : {33, 64, 100}) calls(mixed(alone, 1 + most % 2, size, most, 7), 8, 4, 1, D, 256, "alone and groups");
  }
  g_tight = 0;
  for (int turn = 0; turn < 1300; ++turn) {
    const int heads[][2] = {{1, 1}, {1, 4}, {8, 4}, {2, 8}, {4, 6}, {1, 7}, {3, 1}, {1, 33}, {1, 128}, {16, 1}};
    const int* h = heads[pick(0, 9)];
    const int sq = pick(1, 4), cus = pick(0, 3) ? 256 : pick(1, 300), D = 64 << pick(0, 2);
    calls(any_batch(65536 / (h[0] * h[1] * sq)), h[0], h[1], sq, D, cus, "any");
  }
  CHECK(g_lines > 1000 && g_shares > 1000 && g_tight > 100);
  std::printf("%ld checks passed, %ld lines, %ld shares\n", g_checks, g_lines, g_shares);
  return 0;
}
