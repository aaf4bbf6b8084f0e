// The plan of the attention of requests that share prefixes (kv8_shared.hip): what the
// units of a call are, how their steps are cut into the blocks' segments, and where a
// block leaves its records and the join finds them.  For the kernels, the workspace,
// and a check on the host that every record that is joined has been written.
#pragma once

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstddef>
#include <cstdint>

#include "jfkv.h"

namespace jfkv {
namespace kv8 {
namespace shared {

#define JF_PLAN __host__ __device__ __forceinline__

// Columns of a group, or left over by its tiles, that the groups' kernel walks by rows at
// most (32,768 positions, 32/8 heads of 128: with 48 left over rows take 97 us and tiles
// 91, with 64 94 and 89; 24/4 heads of 256 over 65,536, 64 left over: 105 and 97).
constexpr int kTileRows = 32;
constexpr int kRowWaves = 4;  // of a block of the row walk
constexpr int kMinRows = 1;   // rows per wave below which a unit is not cut (1: 14.2 us, 2: 14.7, 4: 16.0)

// What a kernel takes: the groups' shared positions, the requests' own, or both.
enum Part { kGroups, kOwn, kBoth };

// How a chunk of columns is computed: by rows, one or two sets of 16 columns for all of
// a block's waves, or by tiles, one or two sets for each of eight waves.  (With
// two each LDS operand feeds two products: at d = 128, 256 columns over 65,536 positions
// take 105 us, with one set 126, 1,024 columns 322 and 419.  At d = 256 two do not fit
// into the registers.)
enum Kind { kRows1, kRows2, kTiles1, kTiles2 };
__host__ __device__ constexpr int widest(int D) { return D > 128 ? 128 : 256; }
__host__ __device__ constexpr int width_log2(int kind) {
  return kind == kRows1 ? 4 : kind == kRows2 ? 5 : kind == kTiles1 ? 7 : 8;
}
__host__ __device__ constexpr int width_of(int kind) { return 1 << width_log2(kind); }
__host__ __device__ constexpr int step_log2(int kind) { return kind >= kTiles1 ? 6 : 5; }
__host__ __device__ constexpr int rows_of(int cols) { return cols <= 16 ? kRows1 : kRows2; }
__host__ __device__ constexpr int kind_of(int D, int cols) {
  return cols <= kTileRows ? rows_of(cols) : cols <= 128 || D > 128 ? kTiles1 : kTiles2;
}
// Cost of a step, and of a unit's start and end, in about 0.1 us of a block.  (Half or
// twice the start: 64 requests of 60 positions 37 -> 41 and 37 us, of 4,096 117 -> 118 and
// 120.)
__host__ __device__ constexpr int cost_of(int kind) {
  return kind == kRows1 ? 4 : kind == kRows2 ? 5 : kind == kTiles1 ? 16 : 24;
}
__host__ __device__ constexpr int start_of(int kind) { return kind >= kTiles1 ? 60 : 30; }
// The dearest step of a kernel's units.
__host__ __device__ constexpr int dearest_step(int D, int part) {
  return cost_of(part == kGroups ? kind_of(D, widest(D)) : kRows2);
}
static_assert(cost_of(kRows1) <= cost_of(kRows2) && cost_of(kRows2) <= cost_of(kTiles1) &&
                  cost_of(kTiles1) <= cost_of(kTiles2),
              "dearest_step takes the widest kind for the dearest");
// The least that a share of a unit costs, or a piece of the line for its length.
constexpr int kLeast = cost_of(kRows1) * kRowWaves * kMinRows;

// Blocks of the row walk per CU.  One set of columns leaves room for more, which hides
// more of a unit's start (three in place of two, 32/8 heads of 128: 256 requests of 300
// positions of their own 79 -> 72 us, 64 of 300 40 -> 37; 64 of 4,096 133 -> 137).  A
// kernel that takes groups as well has two: its second walk would spill (16 requests over
// 8,192 shared positions 24.2 -> 26.9 us with three).
__host__ __device__ constexpr int row_blocks(int D, bool one_set) {
  return one_set ? (D > 128 ? 2 : D > 64 ? 3 : 4) : 2;
}

// floor(y / d) for 0 <= y < 2^53 and 0 < d: the nearest quotient of two whole numbers does
// not reach the next whole number.  (Some twenty instructions; a division of 64-bit
// integers has over a hundred.)
JF_PLAN int64_t whole(int64_t y, int64_t d) { return (int64_t)floor((double)y / (double)d); }

// An item of the line: the full chunks of a group's columns over its shared positions
// (items 2 g), the other columns (2 g + 1), or a request's own positions.  Its units are
// its chunks, for each of the KV heads.
struct Item {
  int request;     // the first one, whose table is read
  int col0, cols;  // columns, counted from that request's first
  int lo, hi;      // positions
  int kind;
  JF_PLAN int chunks() const { return (cols - col0 + width_of(kind) - 1) >> width_log2(kind); }
  JF_PLAN int steps() const {
    const int s = step_log2(kind);
    return hi > lo ? ((hi - 1) >> s) - (lo >> s) + 1 : 0;
  }
  // cost of a unit but for its start
  JF_PLAN int64_t work() const { return (int64_t)steps() * cost_of(kind); }
  // a unit's part of the line
  JF_PLAN int64_t span() const {
    const int64_t w = work();
    return w ? start_of(kind) + w : 0;
  }
};

// Items of a kernel, and item i of them.  Args: the call's sizes; Batch: its groups
// (first, shared: their requests and positions; of: a request's) and lengths.
template <int PART, class Args>
JF_PLAN int items_of(const Args& a) {
  return (PART == kOwn ? 0 : 2 * a.G) + (PART == kGroups ? 0 : a.B);
}
template <int D, int PART, class Args, class Batch>
JF_PLAN Item item_of(const Args& a, const Batch& batch, int i) {
  Item t;
  const int pairs = a.gq * a.sq;
  if (PART == kGroups || (PART == kBoth && i < 2 * a.G)) {
    constexpr int W = widest(D);
    const int g = i >> 1;
    t.request = batch.first(g);
    const int cols = batch.valid ? (batch.first(g + 1) - t.request) * pairs : 0;
    const int full = PART == kBoth ? 0 : cols & -W;
    t.col0 = i & 1 ? full : 0;
    t.cols = i & 1 ? cols : full;
    t.kind = PART == kBoth ? rows_of(cols) : kind_of(D, i & 1 ? cols - full : W);
    t.lo = 0, t.hi = t.cols > t.col0 ? batch.shared(g) : 0;
  } else {
    t.request = PART == kOwn ? i : i - 2 * a.G;
    t.col0 = 0, t.cols = pairs;
    t.lo = batch.valid ? batch.shared(batch.of(t.request)) : 0, t.hi = batch.length(t.request);
    t.kind = a.own_kind;
  }
  return t;
}

// Where a chunk of `cols` columns from the request's `col` on has its place for a KV head
// (counted in columns, one chunk after the other in the line's order): its entry of
// `info`, and, with a gap of the widest chunk from each block to the next, its records.
template <class Args>
JF_PLAN int place_of(const Args& a, int request, int col, int cols, int kv) {
  return (request * a.gq * a.sq + col) * a.Hkv + kv * cols;
}

// Steps r0 .. r1 - 1 of an item's unit u, which leaves `records` records, one for each
// block from that of its first step on; on the line the next unit begins at `next`.
struct Cut {
  int u, r0, r1, records;
  int64_t next;
};

// The line: the units follow one another, each with its start's cost, and the line is cut
// into pieces of one length, a block each.  No piece is shorter than a step of any unit:
// between the blocks of a unit's first and last step each then has the beginning of a
// step, and so a record, as cut_line counts them.
template <int D, int PART>
JF_PLAN int64_t piece_of(int64_t line, int blocks) {
  constexpr int least = std::max(kLeast, dearest_step(D, PART));
  return std::max(whole(line, blocks) + 1, (int64_t)least);
}
// The unit of item `it` (which begins at `from`) that place x lies in, and its steps that
// begin in begin .. end - 1, a block's piece of the line that holds x.
JF_PLAN Cut cut_line(const Item& it, int64_t from, int64_t x, const int64_t& begin, int64_t end, int64_t piece) {
  const int cost = cost_of(it.kind), steps = it.steps();
  const int64_t length = it.span(), in = x - from;
  const int u = in < length ? 0 : (int)whole(in, length);
  const int64_t start = x - in + u * length, at = start + start_of(it.kind), work = it.work();
  const auto upto = [&](int64_t y) {  // steps that begin before y
    return (int)whole(std::max(y - at, (int64_t)0) + cost - 1, cost);
  };
  const int r0 = upto(x);
  int r1 = steps, more = 0;
  if (end < at + work) {
    r1 = upto(end);
    // the last step's piece, counted from this block's (each between has a step)
    more = (int)whole(at + work - cost - begin, piece);
  }
  return {u, r0, r1, 1 + more, start + length};
}

// Shares: each unit is cut into equal ones, as many for all units as there are blocks or
// less, a block each.  For few units, items that a block's `window` threads hold, and work
// that a float counts; the line is for the others.
JF_PLAN bool takes_line(int64_t work, int count, int blocks, int items, int window) {
  return 2 * count > blocks || items > window || work >= 0x40000000;
}
// Their length lies between work / blocks and work / (blocks - count): the team'th of
// `teams` lengths to choose from, the last of which is always long enough.
JF_PLAN float share_length(int64_t work, int count, int blocks, int team, int teams) {
  const float low = (float)work / (float)blocks, high = (float)work / (float)(blocks - count) * 1.0001f + 1.0f;
  return fmaxf(low + (high - low) * ((float)team / (teams - 1)), (float)kLeast);
}
// Shares of a unit's work (below 2^31) of at most `most` each.
JF_PLAN int shares(int work, float most) {
  return work ? std::max((int)ceilf((float)work / most), 1) : 0;
}
// Share j of an item whose units have `each`.
JF_PLAN Cut cut_share(const Item& it, int each, int j) {
  const int u = (int)(((float)j + 0.5f) / (float)each), share = j - u * each;  // (both below 2^16)
  const uint32_t steps = it.steps(), size = (steps + each - 1) / (uint32_t)each;
  const int r0 = (int)std::min(share * size, steps), r1 = (int)std::min(r0 + size, steps);
  return {u, r0, r1, (int)((steps + size - 1) / size), 0};
}

// What a segment has besides: its chunk's first column, its KV head, its place.
struct Spot {
  int col, kv, at;
};
template <class Args>
JF_PLAN Spot spot_of(const Args& a, const Item& it, int u) {
  const int chunk = (int)(((float)u + 0.5f) / (float)a.Hkv), kv = u - chunk * a.Hkv;  // (u below 2^17)
  const int col = it.col0 + (chunk << width_log2(it.kind));
  return {col, kv, place_of(a, it.request, col, std::min(width_of(it.kind), it.cols - col), kv)};
}
// Its record of a block, in columns.
template <class Args>
JF_PLAN int64_t record_of(const Args& a, bool own, int block, int at) {
  return (int64_t)(own ? a.own_recs + a.own_gap * block : a.group_gap * block) + at;
}

// What the join asks for: the place of the chunk that holds column `pair` of a request's
// own positions, or of its group's (requests from .. to - 1) shared ones, and the column's
// place in it.
struct Asked {
  int at, in;
};
template <class Args>
JF_PLAN Asked own_of(const Args& a, int b, int pair, int kv) {
  const int pairs = a.gq * a.sq, width = width_of(a.own_kind), col = pair & -width;
  return {place_of(a, b, col, std::min(width, pairs - col), kv), pair - col};
}
template <int D, class Args>
JF_PLAN Asked group_of(const Args& a, bool both, int from, int to, int b, int pair, int kv) {
  constexpr int W = widest(D);
  const int pairs = a.gq * a.sq, cols = (to - from) * pairs;
  const int col = (b - from) * pairs + pair, full = both ? 0 : cols & -W;
  const int begin = col < full ? 0 : full, end = col < full ? full : cols;
  const int width = width_of(both ? rows_of(cols) : kind_of(D, col < full ? W : cols - full));
  const int first = begin + ((col - begin) & -width);  // of its chunk
  return {place_of(a, from, first, std::min(width, end - first), kv), col - first};
}

// How the workspace is laid out: entries, then records.
struct Layout {
  bool both;  // one kernel for groups and requests
  int group_blocks, own_blocks, own_kind, group_gap, own_gap, own_info, own_recs;
  size_t recs, bytes;
};
inline Layout layout_of(const jf_kv_layout& L, int32_t B, int32_t sq, int32_t Hq, bool both, int cus) {
  const int D = L.head_dim, pairs = Hq / L.num_kv_heads * sq, columns = B * Hq * sq;
  Layout p;
  p.both = both;
  p.own_kind = rows_of(pairs);
  p.own_blocks = row_blocks(D, !both && p.own_kind == kRows1) * cus;
  p.group_blocks = both ? p.own_blocks : cus;
  p.group_gap = both ? width_of(kRows2) : widest(D);
  p.own_gap = std::min(pairs, width_of(p.own_kind));
  p.own_info = columns;
  p.own_recs = columns + p.group_blocks * p.group_gap;
  p.recs = ((size_t)columns * 2 * sizeof(int2) + 15) / 16 * 16;
  p.bytes = p.recs + (size_t)(p.own_recs + columns + p.own_blocks * p.own_gap) * (D + 4) * sizeof(float);
  return p;
}
// Whether rows are walked for groups too, in one kernel with the requests' own positions:
// for batches of up to 128 columns (rows against tiles, 32/8 heads of 128, 32 requests:
// over 65,536 positions 70 against 80 us, over 4,096 and 300 of their own 29 against 42;
// 24/4 heads of 256, 21 requests over 32,768: 53 against 55), and for more where columns,
// heads and the table's positions are too few to pay for a kernel of tiles, whose records
// are wider and whose start is longer (64 requests over 4,096: 37 against 58 us, over
// 16,384: 70 both, over 32,768: 107 against 87; 256 over 4,096: 93 against 96, over 8,192:
// 135 against 113; heads of 256, 42 requests: over 4,096 35 against 50, over 16,384 62
// both, over 32,768 97 against 79).
inline bool by_rows(const jf_kv_layout& L, int32_t B, int32_t sq, int32_t Hq, int32_t max_pages) {
  const int64_t columns = (int64_t)B * (Hq / L.num_kv_heads) * sq;
  const int64_t few = L.head_dim > 128 ? 1 << 24 : 1 << 25;
  return columns <= 128 || columns * L.num_kv_heads * ((int64_t)max_pages * L.page_size) <= few;
}

}  // namespace shared
}  // namespace kv8
}  // namespace jfkv
