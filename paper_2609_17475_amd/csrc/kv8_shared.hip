// Decode attention over the 8-bit cache (format: jfkv_kv8.h) of a batch whose requests
// share prefixes: the shared positions of a group are read once for all of its
// requests' queries, each request's own positions for itself, and the parts of a row
// are joined by their log-sum-exps.
//
//   o = sum_j 2^(m_j - M) o_j / sum_j 2^(m_j - M) l_j,   M = max m_j
//
// for parts j with running maximum m_j, sum l_j and unnormalised output o_j (log2
// units), whatever positions each of them covered.
//
// The (request, token, head) triples that read a KV head are the columns of the
// matrix products, 16 to a set, and what kv8_decode.hip says of operands, exponents
// and roundings holds here too.  Two ways to walk: rows of 32 positions, each wave its
// own for up to 32 columns (requests' own positions, small groups; bound by HBM, or by
// latency), and tiles of 64 positions, each wave with columns of its own (large groups;
// bound by the vector work beside the matrix cores, as the chunk attention).  The work
// of a launch is a line of units: for each group its chunks of columns and KV heads,
// then for each request its KV heads; a unit is a run of steps over positions.  The
// line is cut into pieces of equal cost, a block each, wherever that falls; each
// (block, unit) leaves one record, which a last launch joins.  Small batches have one
// kernel before that, large ones a kernel of tiles and one of rows (the registers that
// tiles need leave rows too few waves: 256 requests of 300 positions over 256 shared
// 79 us in one kernel of both, 72 in two).
//
// A step of 64 requests of 200 to 2,000 positions over 32,768 shared (32/8 heads of
// 128) takes 106 us: 59 in the tiles (half of it vector work and matrix products, the
// rest the plan, queries, first tiles, and 35 MB of records), 38 in the rows (4 TB/s),
// 9 in the join; 256 requests over 65,536 350 us, 300 of them in the tiles, 920 TFLOP/s;
// two requests over 4,096 14 us: a plan, a walk and a join, each a chain of latencies.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "jfkv_internal.h"
#include "jfkv_kv8.h"
#include "jfkv_kv8_shared_plan.h"
#include "jfkv_kv8_tiles.h"

namespace jfkv {
namespace {

using namespace kv8;
using namespace kv8::shared;
using tiles::kTile;
using tiles::walk_tiles;

constexpr int kRow = 32;        // positions that a wave of the row walk takes at a time (in one page)
constexpr int kTileWaves = tiles::kWaves;
constexpr int kRowThreads = 64 * kRowWaves, kTileThreads = 64 * kTileWaves;
constexpr float kLn2 = 0.69314718055994530942f;

// Values that are the same in all lanes, to scalar registers.
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ int64_t uniform(int64_t x) {
  return (int64_t)((uint64_t)(uint32_t)uniform((int)(x >> 32)) << 32 | (uint32_t)uniform((int)x));
}

// What a walk reads.  (Kernel arguments of their own: the compiler then knows that no
// store meets them.)
struct Cache {
  const uint8_t *k_codes, *k_exps, *v_codes, *v_exps;
  const uint16_t* q;
  const int32_t* tables;
};
struct Args {
  const int32_t *first, *shared;
  int2* info;    // (first block, records) of each unit
  int B, G, sq, Hq, Hkv, gq, P, block_shift, num_pages, max_pages;
  int own_kind;  // of requests' own units
  int group_gap, own_gap;   // columns from a block's records to the next one's
  int own_info, own_recs;   // where requests' begin (entries, columns; groups' are before)
  float scale_log2;
  uint32_t flip;  // a negative scale negates the queries instead
};

// Groups and lengths, from LDS where they fit.  The groups are valid only if their
// bounds ascend from 0 to B.
typedef const __attribute__((address_space(3))) int32_t* Lds;
struct Batch {
  const int32_t *g_first, *g_shared, *g_lens;
  Lds s_first, s_shared, s_lens;
  int groups, cap;
  bool in_lds, valid;
  __device__ __forceinline__ int first(int g) const { return in_lds ? s_first[g] : g_first[g]; }
  __device__ __forceinline__ int length(int b) const {
    return min(max(in_lds ? s_lens[b] : g_lens[b], 0), cap);
  }
  // the group of request b
  __device__ __forceinline__ int of(int b) const {
    int lo = 0, hi = groups;
    while (hi - lo > 1) {
      const int mid = (lo + hi) / 2;
      if (first(mid) <= b) lo = mid; else hi = mid;
    }
    return lo;
  }
  // Positions that group g's requests share (none for a request alone): those that its
  // first request, whose table is read, has.
  __device__ __forceinline__ int shared(int g) const {
    const int b = first(g);
    if (!valid || first(g + 1) - b < 2) return 0;
    return min(max(in_lds ? s_shared[g] : g_shared[g], 0), length(b));
  }
};

// Where a block is on the line: at x, up to end; the window of items that is summed up
// begins with item `window`.
struct State {
  int64_t x, begin, end, piece;
  int window;
  bool valid, apart;
};
// Steps r0 .. r1 - 1 of a unit: its chunk's first column, KV head and record.
struct Segment {
  Item it;
  int col, kv, r0, r1;
  int64_t rec;
};
// The plan of a block of T threads: which segments it has.  Where units are few, each is
// cut into equal shares, as many for all units as there are blocks, and a block has one
// share; else the units follow one another on a line, each with its start's cost, and
// the line is cut into pieces of one length.  (Two requests over 4,096 positions: 14.7 us
// in shares, 16.7 on the line, where a piece may begin in one unit and end in the next;
// 16 over 8,192: 24.3 and 30.3; four groups of 24: 108 and 115.  What lives from one
// segment to the next is in LDS, so that the walks have the registers.)
template <int T>
struct Plan {
  static constexpr int kTeams = T / 64;
  Args a;
  State state;
  Segment segment;
  int64_t upto[T + 1];  // the line up to the window's item i, itself among it: upto[i + 1]
  Item items[T];
  int64_t sum[kTeams];
  int units[kTeams], starts[kTeams];
  float lengths[kTeams];
  int32_t first[T + 1], shared[T], lens[2 * T];

  __device__ __forceinline__ Batch batch(const Args& g, const int32_t* g_lens, bool valid) const {
    return Batch{g.first, g.shared, g_lens, (Lds)first, (Lds)shared, (Lds)lens, g.G, g.max_pages * g.P,
                 g.G <= T && g.B <= 2 * T, valid};
  }

  // All threads: the block's first segment; false: there is none.
  template <int D, int PART>
  __device__ __forceinline__ bool begin(const Args& g, const int32_t* g_lens) {
    const int tid = threadIdx.x, lane = tid & 63, team = uniform(tid >> 6), blocks = gridDim.x;
    Batch b = batch(g, g_lens, true);
    int bad = 0;
    for (int i = tid; i <= g.G; i += T) {
      const int at = g.first[i];
      bad |= i == 0 ? at != 0 : at < g.first[i - 1];
      if (i == g.G) bad |= at != g.B;
      if (b.in_lds) {
        first[i] = at;
        if (i < g.G) shared[i] = g.shared[i];
      }
    }
    if (b.in_lds)
      for (int i = tid; i < g.B; i += T) lens[i] = g_lens[i];
    b.valid = !__syncthreads_or(bad);

    // all items' work, units and starts
    const int n = items_of<PART>(g);
    int64_t work = 0;
    int count = 0, begins = 0, units_here = 0, work_here = 0;
    Item t = {};
    for (int i = tid; i < n; i += T) {
      t = item_of<D, PART>(g, b, i);
      const int64_t w = t.work();
      const int m = w ? t.chunks() * g.Hkv : 0;
      work += w * m, count += m, begins += m * start_of(t.kind);
      work_here = (int)min(w, (int64_t)0x7fffffff), units_here = m;
      items[tid] = t;
    }
#pragma unroll
    for (int o = 32; o; o >>= 1)
      work += __shfl_xor(work, o), count += __shfl_xor(count, o), begins += __shfl_xor(begins, o);
    if (lane == 0) sum[team] = work, units[team] = count, starts[team] = begins;
    __syncthreads();
    work = 0, count = begins = 0;
#pragma unroll
    for (int w = 0; w < kTeams; ++w) work += sum[w], count += units[w], begins += starts[w];
    work = uniform(work), count = uniform(count), begins = uniform(begins);
    if (count == 0) return false;
    if (takes_line(work, count, blocks, n, T)) {
      if (tid == 0) {
        a = g;
        const int64_t piece = piece_of<D, PART>(work + begins, blocks);
        const int64_t from = blockIdx.x * piece;
        state = State{from, from, min(from + piece, work + begins), piece, -T, b.valid, false};
        upto[T] = 0;  // (no window yet)
      }
      __syncthreads();
      return next<D, PART>(g_lens);
    }

    // Shares: each wave counts those of one length, the least that are not too many are
    // taken.
    const float length = share_length(work, count, blocks, team, kTeams);
    __syncthreads();  // (`units` is written again)
    int many = 0;
    for (int i = lane; i < n; i += 64) {
      const Item u = items[i];
      const int w = (int)u.work();
      if (w) many += shares(w, length) * (u.chunks() * g.Hkv);
    }
#pragma unroll
    for (int o = 32; o; o >>= 1) many += __shfl_xor(many, o);
    if (lane == 0) units[team] = many, lengths[team] = length;
    __syncthreads();
    int pick = kTeams - 1;
#pragma unroll
    for (int w = kTeams - 2; w >= 0; --w)
      if (units[w] <= blocks) pick = w;
    // the block's share: one thread's item has it
    const int each = shares(work_here, lengths[pick]), all = each * units_here;
    int to = all;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int up = __shfl_up(to, o);
      if (lane >= o) to += up;
    }
    if (lane == 63) starts[team] = to;
    if (tid == 0) a = g, state.apart = true, state.valid = b.valid, segment.r0 = segment.r1 = 0;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kTeams; ++w) to += w < team ? starts[w] : 0;
    const int j = (int)blockIdx.x - (to - all);
    if (j >= 0 && j < all) put<D, PART>(g, t, tid, cut_share(t, each, j));
    __syncthreads();
    return uniform(segment.r0) < uniform(segment.r1);
  }

  // The block's segment of item i.
  template <int D, int PART>
  __device__ __forceinline__ void put(const Args& g, const Item& it, int i, const Cut& c) {
    const Spot spot = spot_of(g, it, c.u);
    const bool own = PART == kOwn || (PART == kBoth && i >= 2 * g.G);
    if (c.r0 == 0 && c.r1 > 0) g.info[own ? g.own_info + spot.at : spot.at] = make_int2(blockIdx.x, c.records);
    segment = Segment{it, spot.col, spot.kv, c.r0, c.r1, record_of(g, own, blockIdx.x, spot.at) * (D + 4)};
  }

  // All threads: the block's next segment; false: none is left.
  template <int D, int PART>
  __device__ __forceinline__ bool next(const int32_t* g_lens) {
    if (uniform((int)state.apart)) return false;
    int tid = threadIdx.x;
    asm volatile("" : "+v"(tid));
    const int lane = tid & 63, team = uniform(tid >> 6);
    const int n = uniform(items_of<PART>(a));
    for (;;) {
      const int64_t x = uniform(state.x);
      int window = uniform(state.window);
      if (x >= uniform(state.end)) return false;
      while (x >= uniform(upto[T])) {
        const int64_t carry = uniform(upto[T]);
        window += T;
        if (window >= n) return false;
        const bool mine = window + tid < n;
        if (n > T && mine) items[tid] = item_of<D, PART>(a, batch(a, g_lens, state.valid), window + tid);
        int64_t to = mine ? items[tid].span() * (items[tid].chunks() * a.Hkv) : 0;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
          const int64_t up = __shfl_up(to, o);
          if (lane >= o) to += up;
        }
        if (lane == 63) sum[team] = to;
        __syncthreads();
        to += carry;
#pragma unroll
        for (int w = 0; w < kTeams; ++w) to += w < team ? sum[w] : 0;
        upto[tid + 1] = to;
        if (tid == 0) upto[0] = carry, state.window = window;
        __syncthreads();
      }
      __syncthreads();
      if (x >= upto[tid] && x < upto[tid + 1]) {  // one thread's item
        // the unit, and its steps that begin in the block's piece
        const Item it = items[tid];
        const Cut c = cut_line(it, upto[tid], x, state.begin, state.end, state.piece);
        put<D, PART>(a, it, window + tid, c);
        state.x = c.next;
      }
      __syncthreads();
      if (uniform(segment.r0) < uniform(segment.r1)) return true;  // (else a unit's start alone)
    }
  }

  // The arguments and the segment, in scalar registers.
  __device__ __forceinline__ Args args() const {
    Args f = a;
    f.sq = uniform(f.sq), f.Hq = uniform(f.Hq), f.Hkv = uniform(f.Hkv), f.gq = uniform(f.gq);
    f.P = uniform(f.P), f.block_shift = uniform(f.block_shift), f.num_pages = uniform(f.num_pages);
    f.max_pages = uniform(f.max_pages), f.flip = uniform((int)f.flip);
    f.scale_log2 = __uint_as_float(uniform((int)__float_as_uint(f.scale_log2)));
    return f;
  }
  __device__ __forceinline__ Segment part() const {
    Segment t = segment;
    t.it.request = uniform(t.it.request), t.it.cols = uniform(t.it.cols), t.it.lo = uniform(t.it.lo);
    t.it.hi = uniform(t.it.hi), t.it.kind = uniform(t.it.kind), t.col = uniform(t.col);
    t.kv = uniform(t.kv), t.r0 = uniform(t.r0), t.r1 = uniform(t.r1), t.rec = uniform(t.rec);
    return t;
  }
};

template <int D>
struct Row {
  u32x4 k[2][D / 64], v[2][D / 64];
  uint32_t exps;  // lanes 0, 1: K's exponent bytes of the two tiles; 2, 3: V's
};

// What column `col` of an item's request reads: its query, and how many positions.
template <int D>
__device__ __forceinline__ const uint16_t* query_of(const Args& a, const Cache& in, const Batch& batch,
                                                    const Item& it, int col, int kv, int& see) {
  const int row = col / a.gq;
  see = min(batch.length(it.request + row / a.sq) - a.sq + 1 + row % a.sq, it.hi);
  return in.q + (((size_t)it.request * a.sq + row) * a.Hq + kv * a.gq + col % a.gq) * D;
}

// The pages of an item: constant memory as far as the kernel goes, read by scalar loads.
typedef const __attribute__((address_space(4))) int32_t* Table;
__device__ __forceinline__ Table table_of(const Args& a, const Cache& in, const Item& it) {
  return (Table)(uintptr_t)(in.tables + (size_t)it.request * a.max_pages);
}

// Steps r0 .. r1 - 1 (counted from the item's first) of the chunk of columns from c0 on,
// its record to rec, by rows.
template <int D, bool BF16, int CS, int WAVES, bool ONCE>
__device__ __forceinline__ void walk_rows(const Args& a, const Cache& in, const Batch& batch,
                                          const Item& it, int c0, int kv,
                                          int r0, int r1, float* rec, float* smem) {
  constexpr int C = D / 64;
  constexpr int kPart = D + 4;  // floats of a partial: o, m, l (16-byte rows)
  int tid = threadIdx.x;
  asm volatile("" : "+v"(tid));  // (opaque: what depends on it is not held from one segment to the next)
  __builtin_assume(tid >= 0 && tid < 64 * WAVES);
  const int lane = tid & 63, n = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int P = a.P, ncols = min(16 * CS, it.cols - c0);

  // ---- page walk: the wave takes rows r0 + wave, + WAVES, ...  A row's registers
  // are refilled with the next row, K's as soon as the scores are formed and V's after
  // the value products.  Page IDs are read one turn before the loads.
  const Table table = table_of(a, in, it);
  const uint32_t koff = n * D + 16 * g, voff = lane * 16;
  const int base = it.lo / kRow, last = base + r1 - 1;  // (rows past the end read the last one again)
  auto page_of = [&](int r) { return table[min(r, last) * kRow / P]; };
  auto run_of = [&](int pid) {
    return (size_t)((uint32_t)pid < (uint32_t)a.num_pages ? pid : 0) * a.Hkv + kv;
  };
  // ONCE: no other block reads it, so it does not push out what others read (64 requests
  // of 4,096 positions of their own 137 -> 119 us, of 200 to 2,000 over 32,768 shared 114 -> 106; where
  // all of it stays in the last cache from call to call it costs: 64 of 300 48 -> 50).
  auto load = [](const uint8_t* from) {
    const u32x4* const p = reinterpret_cast<const u32x4*>(from);
    return ONCE ? __builtin_nontemporal_load(p) : *p;
  };
  auto fetch_k = [&](Row<D>& w, int r, int pid) {
    const int slot0 = min(r, last) * kRow % P;
    const size_t run = run_of(pid);
    const uint8_t* kp = in.k_codes + (run * P + slot0) * D;
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int c = 0; c < C; ++c)
        w.k[t][c] = load(kp + koff + t * 16 * D + c * 64);
    const uint8_t* ep = (lane & 2) ? in.v_exps : in.k_exps;
    w.exps = ep[run * (P >> a.block_shift) + ((slot0 + 16 * (lane & 1)) >> a.block_shift)];
  };
  auto fetch_v = [&](Row<D>& w, int r, int pid) {
    const int slot0 = min(r, last) * kRow % P;
    const uint8_t* vp = in.v_codes + (run_of(pid) * P + slot0) * D;
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int c = 0; c < C; ++c)
        w.v[t][c] = load(vp + voff + t * 16 * D + c * 1024);
  };

  Row<D> w;
  int r = base + r0 + wave;
  int pid = page_of(r), ahead = page_of(r + WAVES);
  fetch_k(w, r, pid);
  fetch_v(w, r, pid);

  // ---- queries as B operands: column n of each set, dims 64 c + 16 g + 8 j .., in
  // registers or, where they would fill them, in LDS
  constexpr bool kQLds = CS > 1;
  int see[CS], least = 0x7fffffff;  // positions the columns' queries see
  u32x4 qf[CS][C][2];
  u32x4* const s_q = reinterpret_cast<u32x4*>(smem);
  __syncthreads();  // (LDS still holds what was before)
#pragma unroll
  for (int cs = 0; cs < CS; ++cs) {
    const int col = c0 + min(16 * cs + n, ncols - 1);  // (columns without a query repeat the last one)
    const uint16_t* const qp = query_of<D>(a, in, batch, it, col, kv, see[cs]);
    least = min(least, see[cs]);
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int j = 0; j < 2; ++j)
        if (!kQLds || wave == (cs * C + c) % WAVES) {
          const u32x4 x = *reinterpret_cast<const u32x4*>(qp + 64 * c + 16 * g + 8 * j) ^ a.flip;
          if (kQLds)
            s_q[64 * ((cs * C + c) * 2 + j) + lane] = x;
          else
            qf[cs][c][j] = x;
        }
  }
#pragma unroll
  for (int o = 1; o < 16; o <<= 1) least = min(least, __shfl_xor(least, o));
  int masked = least - kRow + 1;  // the first position at which a row is masked
  asm("" : "+v"(masked));         // (in a vector register, as in the tiles' walk)
  if (kQLds) __syncthreads();

  f32x4 acc[CS][C][4] = {};
  float m[CS], l[CS];
#pragma unroll
  for (int cs = 0; cs < CS; ++cs) m[cs] = -INFINITY, l[cs] = 0.0f;
  int e_ref = 0, e_top = -1000;

  // scores of a row in log2 units, and the exponents of its values
  auto scores = [&](const Row<D>& w, int r, float (&s)[CS][2][4], int (&ev)[2]) {
    const int pos0 = r * kRow;
    f32x4 x[2][CS] = {};
    int ql = lane;
    asm volatile("" : "+v"(ql));  // (opaque: LDS is not read ahead of the page walk)
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        u32x4 qc[CS];
#pragma unroll
        for (int cs = 0; cs < CS; ++cs)
          qc[cs] = kQLds ? s_q[64 * ((cs * C + c) * 2 + j) + ql] : qf[cs][c][j];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          const u32x4 k = widen8<BF16>(w.k[t][c][2 * j], w.k[t][c][2 * j + 1]);
#pragma unroll
          for (int cs = 0; cs < CS; ++cs) x[t][cs] = mma<BF16>(k, qc[cs], x[t][cs]);
        }
      }
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const float f = a.scale_log2 * power2(__builtin_amdgcn_readlane((int)w.exps, t) - 127);
      ev[t] = __builtin_amdgcn_readlane((int)w.exps, 2 + t) - 127;
#pragma unroll
      for (int cs = 0; cs < CS; ++cs)
#pragma unroll
        for (int i = 0; i < 4; ++i) s[cs][t][i] = x[t][cs][i] * f;
    }
    if (pos0 >= masked || pos0 < it.lo) {
      // positions that a query does not see, slots not written yet, and slots before
      // the item's (their codes, a NaN among them, and exponents are not looked at)
#pragma unroll
      for (int cs = 0; cs < CS; ++cs)
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int pos = pos0 + 16 * t + 4 * g + i;
            if (pos >= see[cs] || pos < it.lo) s[cs][t][i] = -INFINITY;
          }
      if (pos0 + 16 >= it.hi) ev[1] = ev[0];
      if (pos0 + 16 <= it.lo) ev[0] = ev[1];
    }
  };
  auto rescale = [&](int cs, float f) {
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int dt = 0; dt < 4; ++dt) acc[cs][c][dt] *= f;
  };
  // e_ref such that lo .. hi lie in its window
  auto refer = [&](int lo, int hi) {
    e_top = max(e_top, hi);
    if (lo >= e_ref && hi <= e_ref + kRefMax) return;
    const int e = max(max(hi - kRefMax, lo - 4), e_top - kRefFloor);
    const float f = reference_step(e_ref, e);
#pragma unroll
    for (int cs = 0; cs < CS; ++cs) rescale(cs, f);
    e_ref = e;
  };
  auto attend = [&](Row<D>& w, int r, const float (&s)[CS][2][4], const int (&ev)[2]) {
    const int pos0 = r * kRow;
    float top[CS];
    bool raise = false;
#pragma unroll
    for (int cs = 0; cs < CS; ++cs) {
      top[cs] = larger(larger(larger(s[cs][0][0], s[cs][0][1]), s[cs][0][2]), s[cs][0][3]);
#pragma unroll
      for (int i = 0; i < 4; ++i) top[cs] = larger(top[cs], s[cs][1][i]);
      raise |= top[cs] > m[cs] + kMargin;
    }
    if (__any(raise)) {
#pragma unroll
      for (int cs = 0; cs < CS; ++cs) {
        const float mn = fmaxf(m[cs], col_max(top[cs]));
        const float f = m[cs] == -INFINITY ? 0.0f : exp2_(m[cs] - mn);
        l[cs] *= f;
        rescale(cs, f);
        m[cs] = mn;
      }
    }
    if (pos0 + kRow > it.hi || pos0 < it.lo) {  // slots that are not the item's: zeros (their codes may be NaN)
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const int at = pos0 + 16 * t + 4 * g;
        const int above = min(max(it.hi - at, 0), 4), below = min(max(it.lo - at, 0), 4);
        const uint32_t keep = (above ? 0xffffffffu >> (8 * (4 - above)) : 0u) &
                              (below < 4 ? 0xffffffffu << (8 * below) : 0u);
#pragma unroll
        for (int c = 0; c < C; ++c) w.v[t][c] &= keep;
      }
    }
    // both tiles with one reference, or one after the other where their exponents are
    // too far apart for that
    int lo = min(ev[0], ev[1]), hi = max(ev[0], ev[1]);
    const int parts = hi - lo <= kRefMax ? 1 : 2;
    for (int part = 0; part < parts; ++part) {
      if (parts > 1) lo = hi = part ? ev[1] : ev[0];
      refer(lo, hi);
      u32x4 pf[CS];
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const bool here = parts == 1 || part == t;
        const float by = (float)(ev[t] - e_ref);
#pragma unroll
        for (int cs = 0; cs < CS; ++cs) {
          const float mu = m[cs] == -INFINITY ? 0.0f : m[cs];
          float p[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) p[i] = exp2_(s[cs][t][i] - mu + by);
          if (here) {
            if (ev[t] - e_ref >= -kRefMax) {
              l[cs] = fmaf((p[0] + p[1]) + (p[2] + p[3]), power2(e_ref - ev[t]), l[cs]);
            } else {  // (far below the largest values: P may vanish, l must not)
              for (int i = 0; i < 4; ++i) l[cs] += exp2_(s[cs][t][i] - mu);
            }
          }
          pf[cs][2 * t] = here ? narrow2<false>(p[0], p[1]) : 0u;
          pf[cs][2 * t + 1] = here ? narrow2<false>(p[2], p[3]) : 0u;
        }
      }
#pragma unroll
      for (int c = 0; c < C; ++c)
#pragma unroll
        for (int dt = 0; dt < 4; ++dt) {
          // (opaque: widened ahead of the loop over the parts, all operands would be
          // held at once)
          uint32_t v0 = w.v[0][c][dt], v1 = w.v[1][c][dt];
          asm volatile("" : "+v"(v0), "+v"(v1));
          const u32x4 v = widen8<false>(v0, v1);
#pragma unroll
          for (int cs = 0; cs < CS; ++cs) acc[cs][c][dt] = mma<false>(v, pf[cs], acc[cs][c][dt]);
        }
    }
  };

  for (; r <= last; r += WAVES) {
    const bool on = (uint32_t)pid < (uint32_t)a.num_pages;
    float s[CS][2][4];
    int ev[2];
    scores(w, r, s, ev);
    fetch_k(w, r + WAVES, ahead);
    if (on) attend(w, r, s, ev);
    fetch_v(w, r + WAVES, ahead);
    pid = ahead;
    ahead = page_of(r + 2 * WAVES);
  }

  // ---- merge the waves in LDS, one set of columns after the other: o (units 1), m, l
  const int wide = min(16, ncols) * kPart;  // floats of a wave
#pragma unroll
  for (int cs = 0; cs < CS; ++cs) {
    const int here = min(16, ncols - 16 * cs);  // columns of the set
    const float den = col_sum(l[cs]);
    float* const mine = smem + wave * wide + n * kPart;
    if (kQLds || cs) __syncthreads();  // (LDS still holds the queries or the last set)
    if (n < here) {
      const float f = __builtin_ldexpf(1.0f, e_ref);
#pragma unroll
      for (int c = 0; c < C; ++c)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          *reinterpret_cast<f32x4*>(mine + 64 * c + 16 * g + 4 * i) =
              f32x4{acc[cs][c][0][i], acc[cs][c][1][i], acc[cs][c][2][i], acc[cs][c][3][i]} * f;
      if (g == 0) mine[D] = m[cs], mine[D + 1] = den;
    }
    __syncthreads();
    for (int i = tid; i < here * (D / 4); i += 64 * WAVES) {
      const int at = i / (D / 4), d4 = i % (D / 4);
      const float* const part = smem + at * kPart;
      float mw[WAVES], M = -INFINITY, sum = 0.0f;
#pragma unroll
      for (int w = 0; w < WAVES; ++w) {
        mw[w] = part[w * wide + D];
        M = fmaxf(M, mw[w]);
      }
      f32x4 num = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int w = 0; w < WAVES; ++w) {
        const float f = mw[w] == -INFINITY ? 0.0f : exp2_(mw[w] - M);
        num += *reinterpret_cast<const f32x4*>(part + w * wide + 4 * d4) * f;
        sum = fmaf(f, part[w * wide + D + 1], sum);
      }
      float* const to = rec + (size_t)(16 * cs + at) * kPart;
      *reinterpret_cast<f32x4*>(to + 4 * d4) = num;
      if (d4 == 0) *reinterpret_cast<f32x2*>(to + D) = f32x2{M, sum};
    }
  }
}

// The same by tiles.
template <int D, bool BF16, int NC>
__device__ __forceinline__ void walk_columns(const Args& a, const Cache& in, const Batch& batch,
                                             const Item& it, int c0,
                                             int kv, int j0, int j1, float* rec, float* smem) {
  constexpr int C = D / 64;
  int tid = threadIdx.x;
  asm volatile("" : "+v"(tid));
  __builtin_assume(tid >= 0 && tid < kTileThreads);
  const int lane = tid & 63, n = lane & 15, g = lane >> 4;
  const int wave = uniform(tid >> 6);
  const int wcol = c0 + wave * 16 * NC;
  const bool active = wcol < it.cols;
  int see[NC], least = 0x7fffffff;
  u32x4 qf[NC][C][2];
  __syncthreads();  // (LDS still holds what was before)
#pragma unroll
  for (int cs = 0; cs < NC; ++cs) {  // (columns past the end repeat the last)
    const uint16_t* const qp = query_of<D>(a, in, batch, it, min(wcol + 16 * cs + n, it.cols - 1), kv, see[cs]);
    least = min(least, see[cs]);
    tiles::load_q<C, BF16>(qf[cs], qp, g, a.flip);
  }
#pragma unroll
  for (int o = 1; o < 16; o <<= 1) least = min(least, __shfl_xor(least, o));
  f32x4 acc[NC][C][4] = {};
  float m[NC], l[NC];
#pragma unroll
  for (int cs = 0; cs < NC; ++cs) m[cs] = -INFINITY, l[cs] = 0.0f;
  int e_ref = 0, e_top = -1000;
  // (the first position at which a tile is masked, in a vector register: with a scalar
  // branch around the masks the compiler holds more at once, and spills)
  int masked = least - kTile + 1;
  asm("" : "+v"(masked));
  const struct {
    int masked;
    const int (&see)[NC];
    __device__ __forceinline__ bool hides_some(int pos0) const { return pos0 >= masked; }
    __device__ __forceinline__ bool hides(int cs, int pos) const { return pos >= see[cs]; }
  } sees{masked, see};
  walk_tiles<D, BF16, NC>(in.k_codes, in.k_exps, in.v_codes, in.v_exps,
                          tid, table_of(a, in, it), a.Hkv, kv, a.P, a.block_shift, a.num_pages,
                          it.hi, j0, j1, a.scale_log2, qf, sees, active, reinterpret_cast<u32x4*>(smem),
                          acc, m, l, e_ref, e_top);
  if (!active) return;
  const float unit = __builtin_ldexpf(1.0f, e_ref);
#pragma unroll
  for (int cs = 0; cs < NC; ++cs) {
    const float den = col_sum(l[cs]);
    const int at = wave * 16 * NC + 16 * cs + n;
    if (c0 + at >= it.cols) continue;
    float* const to = rec + (size_t)at * (D + 4);
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        *reinterpret_cast<f32x4*>(to + 64 * c + 16 * g + 4 * i) =
            f32x4{acc[cs][c][0][i], acc[cs][c][1][i], acc[cs][c][2][i], acc[cs][c][3][i]} * unit;
    if (g == 0) *reinterpret_cast<f32x2*>(to + D) = f32x2{m[cs], den};
  }
}

// Requests' own positions (SETS of 16 columns), and groups' in small batches.
template <int D, bool BF16, int PART, int SETS>
__global__ __launch_bounds__(kRowThreads, row_blocks(D, PART == kOwn && SETS == 1)) void kv8_shared_rows_kernel(
    const uint8_t* __restrict__ k_codes, const uint8_t* __restrict__ k_exps,
    const uint8_t* __restrict__ v_codes, const uint8_t* __restrict__ v_exps,
    const uint16_t* __restrict__ q, const int32_t* __restrict__ tables,
    const int32_t* __restrict__ lens, float* __restrict__ recs, const Args a) {
  extern __shared__ __align__(1024) float smem[];
  __shared__ Plan<kRowThreads> plan;
  const Cache in{k_codes, k_exps, v_codes, v_exps, q, tables};
  for (bool more = plan.begin<D, PART>(a, lens); more; more = plan.next<D, PART>(lens)) {
    const Args f = plan.args();
    const Segment t = plan.part();
    const Batch batch = plan.batch(f, lens, plan.state.valid);
    if (PART == kOwn ? SETS == 1 : t.it.kind == kRows1)
      walk_rows<D, BF16, 1, kRowWaves, PART == kOwn>(f, in, batch, t.it, t.col, t.kv, t.r0, t.r1, recs + t.rec, smem);
    else
      walk_rows<D, BF16, 2, kRowWaves, PART == kOwn>(f, in, batch, t.it, t.col, t.kv, t.r0, t.r1, recs + t.rec, smem);
  }
}

// Groups' shared positions.
template <int D, bool BF16>
__global__ __launch_bounds__(kTileThreads) void kv8_shared_groups_kernel(
    const uint8_t* __restrict__ k_codes, const uint8_t* __restrict__ k_exps,
    const uint8_t* __restrict__ v_codes, const uint8_t* __restrict__ v_exps,
    const uint16_t* __restrict__ q, const int32_t* __restrict__ tables,
    const int32_t* __restrict__ lens, float* __restrict__ recs, const Args a) {
  extern __shared__ __align__(1024) float smem[];
  __shared__ Plan<kTileThreads> plan;
  const Cache in{k_codes, k_exps, v_codes, v_exps, q, tables};
  for (bool more = plan.begin<D, kGroups>(a, lens); more; more = plan.next<D, kGroups>(lens)) {
    const Args f = plan.args();
    const Segment t = plan.part();
    const Batch batch = plan.batch(f, lens, plan.state.valid);
    constexpr int kMost = widest(D) / 128;
    float* const rec = recs + t.rec;
    if (t.it.kind == kRows1)
      walk_rows<D, BF16, 1, kTileWaves, false>(f, in, batch, t.it, t.col, t.kv, t.r0, t.r1, rec, smem);
    else if (t.it.kind == kRows2)
      walk_rows<D, BF16, 2, kTileWaves, false>(f, in, batch, t.it, t.col, t.kv, t.r0, t.r1, rec, smem);
    else if (kMost == 1 || t.it.kind == kTiles1)
      walk_columns<D, BF16, 1>(f, in, batch, t.it, t.col, t.kv, t.r0, t.r1, rec, smem);
    else
      walk_columns<D, BF16, kMost>(f, in, batch, t.it, t.col, t.kv, t.r0, t.r1, rec, smem);
  }
}

// Joins the records of a row: a block takes 64 runs of four dims of the rows of one
// (request, KV head), each wave every fourth record.
constexpr int kJoinWaves = 4;
template <int D, bool BF16>
__global__ __launch_bounds__(64 * kJoinWaves) void kv8_shared_join_kernel(
    const float* __restrict__ recs, const int32_t* __restrict__ lens, uint16_t* __restrict__ out,
    float* __restrict__ lse, const Args a, bool both, int group_blocks, int own_blocks) {
  constexpr int kPart = D + 4, kAt = 4;
  __shared__ f32x4 s_num[kJoinWaves][64];
  __shared__ f32x2 s_ml[kJoinWaves][64];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int kv = blockIdx.y, b = blockIdx.z, gq = a.gq, pairs = gq * a.sq;

  Batch batch{a.first, a.shared, lens, nullptr, nullptr, nullptr, a.G, a.max_pages * a.P, false, true};
  const int i = blockIdx.x * 64 + lane, pair = min(i / (D / 4), pairs - 1), d4 = i % (D / 4);
  // what does not wait for the groups: the request's own records
  const Asked mine = own_of(a, b, pair, kv);
  const int2 own = a.info[a.own_info + mine.at];  // (nothing of use where it has none)
  const int len = batch.length(b);
  int group, from, to, shared;  // the request's group, its requests and shared positions
  if (a.G < 64) {       // a lane for each bound: two loads in a row less (16 requests over 8,192 positions 23.8 -> 23.5 us)
    const int at = lane <= a.G ? a.first[lane] : 0, before = __shfl_up(at, 1);
    const int most = lane < a.G ? a.shared[lane] : 0;
    batch.valid = !__any(lane <= a.G && (lane == 0 ? at != 0 : at < before || (lane == a.G && at != a.B)));
    group = max(__popcll(__ballot(lane < a.G && at <= b)) - 1, 0);
    from = __builtin_amdgcn_readlane(at, group), to = __builtin_amdgcn_readlane(at, group + 1);
    const int first_most = __builtin_amdgcn_readlane(most, group);
    shared = batch.valid && to - from > 1 ? min(max(first_most, 0), batch.length(from)) : 0;
  } else {
    int bad = 0;
    for (int i = tid; i <= a.G; i += 64 * kJoinWaves) {
      const int at = a.first[i];
      bad |= i == 0 ? at != 0 : at < a.first[i - 1];
      if (i == a.G) bad |= at != a.B;
    }
    batch.valid = !__syncthreads_or(bad);
    group = batch.valid ? batch.of(b) : 0;
    from = batch.first(group), to = batch.first(group + 1);
    shared = batch.shared(group);
  }

  f32x4 num = {0.0f, 0.0f, 0.0f, 0.0f};
  float M = -INFINITY, den = 0.0f;
  auto add = [&](int from, int gap, int count) {  // (columns)
    for (int r = wave; r < count; r += kJoinWaves * kAt) {
      f32x4 o[kAt];
      f32x2 ml[kAt];
#pragma unroll
      for (int k = 0; k < kAt; ++k) {
        const float* p = recs + (int64_t)(from + min(r + k * kJoinWaves, count - 1) * gap) * kPart;
        o[k] = *reinterpret_cast<const f32x4*>(p + 4 * d4);
        ml[k] = *reinterpret_cast<const f32x2*>(p + D);
      }
      float mx = M;
#pragma unroll
      for (int k = 0; k < kAt; ++k) mx = fmaxf(mx, ml[k].x);
      const float f = M == -INFINITY ? 0.0f : exp2_(M - mx);
      num *= f, den *= f;
#pragma unroll
      for (int k = 0; k < kAt; ++k) {
        const float w = r + k * kJoinWaves >= count || ml[k].x == -INFINITY ? 0.0f : exp2_(ml[k].x - mx);
        num += o[k] * w;
        den = fmaf(w, ml[k].y, den);
      }
      M = mx;
    }
  };
  if (shared > 0) {
    const Asked ours = group_of<D>(a, both, from, to, b, pair, kv);
    const int2 in = a.info[ours.at];
    add(ours.at + in.x * a.group_gap + ours.in, a.group_gap, min(in.y, group_blocks));
  }
  if (len > shared)
    add(a.own_recs + mine.at + own.x * a.own_gap + mine.in, a.own_gap, min(own.y, own_blocks));
  s_num[wave][lane] = num;
  s_ml[wave][lane] = f32x2{M, den};
  __syncthreads();
  if (wave || i >= pairs * (D / 4)) return;
  float mx = -INFINITY;
#pragma unroll
  for (int w = 0; w < kJoinWaves; ++w) mx = fmaxf(mx, s_ml[w][lane].x);
  num = f32x4{0.0f, 0.0f, 0.0f, 0.0f}, den = 0.0f;
#pragma unroll
  for (int w = 0; w < kJoinWaves; ++w) {
    const f32x2 ml = s_ml[w][lane];
    const float f = ml.x == -INFINITY ? 0.0f : exp2_(ml.x - mx);
    num += s_num[w][lane] * f;
    den = fmaf(f, ml.y, den);
  }
  const float r = den > 0.0f ? 1.0f / den : 0.0f;
  const size_t row = ((size_t)b * a.sq + pair / gq) * a.Hq + kv * gq + pair % gq;
  *reinterpret_cast<uint2*>(out + row * D + 4 * d4) =
      make_uint2(narrow2<BF16>(num.x * r, num.y * r), narrow2<BF16>(num.z * r, num.w * r));
  if (lse && d4 == 0) lse[row] = den > 0.0f ? (mx + __log2f(den)) * kLn2 : -INFINITY;
}

template <int D, bool BF16>
hipError_t launch_t(const Cache& in, const int32_t* lens, const Args& a, const Layout& p, float* recs,
                    void* out, float* lse, hipStream_t stream) {
  auto go = [&](auto kernel, int blocks, int threads, size_t lds) {
    if (lds > 32768) {
      const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel),
                                               hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
      if (e != hipSuccess) return e;
    }
    hipLaunchKernelGGL(kernel, dim3(blocks), dim3(threads), lds, stream, in.k_codes, in.k_exps,
                       in.v_codes, in.v_exps, in.q, in.tables, lens, recs, a);
    return hipGetLastError();
  };
  // (the waves' merge; the queries before it take less)
  const size_t merge = sizeof(float) * kRowWaves * 16 * (D + 4);
  hipError_t e = hipSuccess;
  if (p.both) {
    e = go(kv8_shared_rows_kernel<D, BF16, kBoth, 2>, p.own_blocks, kRowThreads, merge);
  } else {
    e = go(kv8_shared_groups_kernel<D, BF16>, p.group_blocks, kTileThreads,
           std::max(4 * 8 * D * sizeof(u32x4), 2 * merge));
    if (e == hipSuccess)
      e = p.own_kind == kRows1 ? go(kv8_shared_rows_kernel<D, BF16, kOwn, 1>, p.own_blocks, kRowThreads, merge)
                               : go(kv8_shared_rows_kernel<D, BF16, kOwn, 2>, p.own_blocks, kRowThreads, merge);
  }
  if (e != hipSuccess) return e;
  const int runs = a.gq * a.sq * (D / 4);
  hipLaunchKernelGGL((kv8_shared_join_kernel<D, BF16>), dim3((runs + 63) / 64, a.Hkv, a.B),
                     dim3(64 * kJoinWaves), 0, stream, recs, lens, static_cast<uint16_t*>(out), lse,
                     a, p.both, p.group_blocks, p.own_blocks);
  return hipGetLastError();
}

}  // namespace

size_t kv8_shared_bytes(const jf_kv_layout& L, int32_t B, int32_t, int32_t sq, int32_t Hq) {
  return std::max(layout_of(L, B, sq, Hq, true, num_cus()).bytes, layout_of(L, B, sq, Hq, false, num_cus()).bytes);
}

hipError_t launch_kv8_shared(const jf_kv_layout& L, const jf_kv_pool_ptrs& pool, bool bf16,
                             const void* q, int32_t B, int32_t sq, int32_t Hq,
                             const int32_t* block_tables, int32_t max_pages, const int32_t* seq_lens,
                             const int32_t* group_start, const int32_t* shared_lens, int32_t G,
                             float softmax_scale, void* ws, void* out, float* lse,
                             hipStream_t stream) {
  const Layout p = layout_of(L, B, sq, Hq, by_rows(L, B, sq, Hq, max_pages), num_cus());
  int shift = 0;
  while ((1 << shift) < L.group_size) ++shift;
  const Cache in{static_cast<const uint8_t*>(pool.k_codes), static_cast<const uint8_t*>(pool.k_meta),
                 static_cast<const uint8_t*>(pool.v_codes), static_cast<const uint8_t*>(pool.v_meta),
                 static_cast<const uint16_t*>(q), block_tables};
  Args a{};
  a.first = group_start, a.shared = shared_lens, a.info = static_cast<int2*>(ws);
  a.B = B, a.G = G, a.sq = sq, a.Hq = Hq, a.Hkv = L.num_kv_heads, a.gq = Hq / L.num_kv_heads, a.P = L.page_size;
  a.block_shift = shift, a.num_pages = L.num_pages, a.max_pages = max_pages;
  a.own_kind = p.own_kind, a.group_gap = p.group_gap, a.own_gap = p.own_gap;
  a.own_info = p.own_info, a.own_recs = p.own_recs;
  a.scale_log2 = std::fabs(softmax_scale) * tiles::kLog2e;
  a.flip = softmax_scale < 0.0f ? 0x80008000u : 0u;
  float* const recs = reinterpret_cast<float*>(static_cast<uint8_t*>(ws) + p.recs);
  auto go = [&](auto fn) { return fn(in, seq_lens, a, p, recs, out, lse, stream); };
  if (L.head_dim == 64) return bf16 ? go(launch_t<64, true>) : go(launch_t<64, false>);
  if (L.head_dim == 128) return bf16 ? go(launch_t<128, true>) : go(launch_t<128, false>);
  return bf16 ? go(launch_t<256, true>) : go(launch_t<256, false>);
}

}  // namespace jfkv
