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
// and roundings holds here too; with more sets per wave a widened code serves more
// products.  The work is a line of units: for each group its chunks of columns and KV
// heads, then for each request its own positions and KV heads; a unit is a run of rows
// of 32 positions.  The line is cut into pieces of equal cost, a block each, wherever
// that falls, so that all CUs end together and products (groups) meet loads (requests);
// each (block, unit) leaves one record, which a second launch joins.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "jfkv_internal.h"
#include "jfkv_kv8.h"

namespace jfkv {
namespace {

using namespace kv8;

constexpr int kWaves = 8;
constexpr int kThreads = 64 * kWaves;
constexpr int kRow = 32;       // positions a wave takes at a time (in one page)
constexpr int kMinRows = 3;    // rows per wave below which a unit is not cut
constexpr int kGroupsLds = 512;
constexpr float kLn2 = 0.69314718055994530942f;

// Sets of 16 columns of a chunk: what the accumulators leave room for.
template <int D>
constexpr int max_sets() {
  return 2;
}
__host__ __device__ constexpr int sets_for(int D, int cols) {
  return cols <= 16 ? 1 : 2;
}
// Cost of a row of 32 positions by its sets.
__host__ __device__ constexpr int row_cost(int sets) { return sets > 2 ? 3 : 2; }

// Values that are the same in all lanes, to scalar registers.
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ int64_t uniform(int64_t x) {
  return (int64_t)((uint64_t)(uint32_t)uniform((int)(x >> 32)) << 32 | (uint32_t)uniform((int)x));
}

// What a walk reads.  (Kernel arguments of their own: the compiler then knows that no
// store meets them, and reads the tables by scalar loads.)
struct Cache {
  const uint8_t *k_codes, *k_exps, *v_codes, *v_exps;
  const uint16_t* q;
  const int32_t *tables, *lens;
};
struct Args {
  const int32_t *first, *shared;
  int2* info;     // (first record, records) of each unit: groups', then requests'
  int B, G, sq, Hq, Hkv, P, block_shift, num_pages, max_pages;
  int group_units, chunks, own_cols;  // chunks and columns of a request's own units
  int64_t own_recs;                   // where requests' records begin (floats)
  float scale_log2;
};

// The groups, from LDS where they fit: valid only if their bounds ascend from 0 to B.
struct Groups {
  const int32_t *first, *shared;
  int n;
  bool valid;
  // the group of request b
  __device__ __forceinline__ int of(int b) const {
    int lo = 0, hi = n;
    while (hi - lo > 1) {
      const int mid = (lo + hi) / 2;
      if (first[mid] <= b) lo = mid; else hi = mid;
    }
    return lo;
  }
};

__device__ __forceinline__ int length_of(const Args& a, const int32_t* lens, int b) {
  return min(max(lens[b], 0), a.max_pages * a.P);
}
// Positions that group g's requests share (none for a request alone): those that its
// first request, whose table is read, has.
__device__ __forceinline__ int shared_of(const Args& a, const int32_t* lens, const Groups& gr, int g) {
  if (!gr.valid || gr.first[g + 1] - gr.first[g] < 2) return 0;
  return min(max(gr.shared[g], 0), length_of(a, lens, gr.first[g]));
}
__device__ __forceinline__ int own_start(const Args& a, const int32_t* lens, const Groups& gr, int b) {
  return gr.valid ? shared_of(a, lens, gr, gr.of(b)) : 0;
}

// An item of the line: a group's shared positions or a request's own ones.
struct Item {
  int request, requests;  // the first one, whose table is read, and how many
  int lo, hi;             // positions
  int sets, chunks, rows;
  int unit;               // number of its first unit
};
template <int D>
__device__ __forceinline__ Item item_of(const Args& a, const int32_t* lens, const Groups& gr, int i) {
  Item t;
  const int pairs = a.Hq / a.Hkv * a.sq;
  if (i < a.G) {
    t.request = gr.valid ? gr.first[i] : 0;
    t.requests = gr.valid ? gr.first[i + 1] - t.request : 0;
    t.lo = 0, t.hi = shared_of(a, lens, gr, i);
    t.sets = sets_for(D, t.requests * pairs);
    t.chunks = (t.requests * pairs + 16 * t.sets - 1) / (16 * t.sets);
    t.unit = (t.request * pairs / (16 * max_sets<D>()) + i) * a.Hkv;
  } else {
    t.request = i - a.G, t.requests = 1;
    t.lo = own_start(a, lens, gr, t.request), t.hi = length_of(a, lens, t.request);
    t.sets = sets_for(D, a.own_cols);
    t.chunks = a.chunks;
    t.unit = a.group_units + t.request * a.chunks * a.Hkv;
  }
  t.rows = t.hi > t.lo ? (t.hi + kRow - 1) / kRow - t.lo / kRow : 0;
  return t;
}
__device__ __forceinline__ int64_t work_of(const Args& a, const Item& t) {
  return (int64_t)t.rows * row_cost(t.sets) * t.chunks * a.Hkv;
}

template <int D>
struct Row {
  u32x4 k[2][D / 64], v[2][D / 64];
  uint32_t exps;  // lanes 0, 1: K's exponent bytes of the two tiles; 2, 3: V's
};

// Rows r0 .. r1 - 1 (counted from the item's first) of one unit: its record to rec.
template <int D, bool BF16, int CS>
__device__ __forceinline__ void walk(const Args& a, const Cache& in, const Item& it, int chunk, int kv, int r0, int r1,
                                     float* rec, float* smem) {
  constexpr int C = D / 64;
  constexpr int kPart = D + 4;  // floats of a partial: o, m, l (16-byte rows)
  const int tid = threadIdx.x, lane = tid & 63, n = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int gq = a.Hq / a.Hkv, P = a.P;
  const int c0 = chunk * 16 * CS, ncols = min(16 * CS, it.requests * a.sq * gq - c0);

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
    const int row = col / gq, head = kv * gq + col % gq, b = it.request + row / a.sq;
    see[cs] = min(length_of(a, in.lens, b) - a.sq + 1 + row % a.sq, it.hi);
    least = min(least, see[cs]);
    const uint16_t* qp = in.q + (((size_t)it.request * a.sq + row) * a.Hq + head) * D;
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int j = 0; j < 2; ++j)
        if (!kQLds || wave == (cs * C + c) % kWaves) {
          const u32x4 x = *reinterpret_cast<const u32x4*>(qp + 64 * c + 16 * g + 8 * j);
          if (kQLds)
            s_q[64 * ((cs * C + c) * 2 + j) + lane] = x;
          else
            qf[cs][c][j] = x;
        }
  }
#pragma unroll
  for (int o = 1; o < 16; o <<= 1) least = min(least, __shfl_xor(least, o));
  if (kQLds) __syncthreads();

  f32x4 acc[CS][C][4] = {};
  float m[CS], l[CS];
#pragma unroll
  for (int cs = 0; cs < CS; ++cs) m[cs] = -INFINITY, l[cs] = 0.0f;
  int e_ref = 0, e_top = -1000;

  // ---- page walk: the wave takes rows r0 + wave, + kWaves, ...  A row's registers
  // are refilled with the next row, K's as soon as the scores are formed and V's after
  // the value products.  Page IDs are read one turn before the loads.
  const int32_t* const table = in.tables + (size_t)it.request * a.max_pages;
  const uint32_t koff = n * D + 16 * g, voff = lane * 16;
  const int base = it.lo / kRow, last = base + r1 - 1;  // (rows past the end read the last one again)
  auto page_of = [&](int r) { return uniform(table[min(r, last) * kRow / P]); };
  auto run_of = [&](int pid) {
    return (size_t)((uint32_t)pid < (uint32_t)a.num_pages ? pid : 0) * a.Hkv + kv;
  };
  auto fetch_k = [&](Row<D>& w, int r, int pid) {
    const int slot0 = min(r, last) * kRow % P;
    const size_t run = run_of(pid);
    const uint8_t* kp = in.k_codes + (run * P + slot0) * D;
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int c = 0; c < C; ++c)
        w.k[t][c] = *reinterpret_cast<const u32x4*>(kp + koff + t * 16 * D + c * 64);
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
        w.v[t][c] = *reinterpret_cast<const u32x4*>(vp + voff + t * 16 * D + c * 1024);
  };

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
    if (pos0 + kRow > least || pos0 < it.lo) {
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

  {
    Row<D> w;
    int r = base + r0 + wave;
    int pid = page_of(r), ahead = page_of(r + kWaves);
    fetch_k(w, r, pid);
    fetch_v(w, r, pid);
    for (; r <= last; r += kWaves) {
      const bool on = (uint32_t)pid < (uint32_t)a.num_pages;
      float s[CS][2][4];
      int ev[2];
      scores(w, r, s, ev);
      fetch_k(w, r + kWaves, ahead);
      if (on) attend(w, r, s, ev);
      fetch_v(w, r + kWaves, ahead);
      pid = ahead;
      ahead = page_of(r + 2 * kWaves);
    }
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
    for (int i = tid; i < here * (D / 4); i += kThreads) {
      const int at = i / (D / 4), d4 = i % (D / 4);
      const float* const part = smem + at * kPart;
      float mw[kWaves], M = -INFINITY, sum = 0.0f;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) {
        mw[w] = part[w * wide + D];
        M = fmaxf(M, mw[w]);
      }
      f32x4 num = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int w = 0; w < kWaves; ++w) {
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

template <int D, bool BF16>
__global__ __launch_bounds__(kThreads) void kv8_shared_kernel(
    const uint8_t* __restrict__ k_codes, const uint8_t* __restrict__ k_exps,
    const uint8_t* __restrict__ v_codes, const uint8_t* __restrict__ v_exps,
    const uint16_t* __restrict__ q, const int32_t* __restrict__ tables,
    const int32_t* __restrict__ lens, float* __restrict__ recs, const Args a) {
  extern __shared__ __align__(16) float smem[];
  __shared__ int64_t s_wave[kWaves], s_upto[kThreads + 1], s_start;
  __shared__ int s_item;
  __shared__ int32_t s_first[kGroupsLds + 1], s_shared[kGroupsLds];
  const Cache in{k_codes, k_exps, v_codes, v_exps, q, tables, lens};
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;

  // ---- the groups
  Groups gr{a.first, a.shared, a.G, true};
  int bad = 0;
  for (int i = tid; i <= a.G; i += kThreads) {
    const int at = a.first[i];
    bad |= i == 0 ? at != 0 : at < a.first[i - 1];
    if (i == a.G) bad |= at != a.B;
    if (a.G <= kGroupsLds) {
      s_first[i] = at;
      if (i < a.G) s_shared[i] = a.shared[i];
    }
  }
  gr.valid = !__syncthreads_or(bad);
  if (a.G <= kGroupsLds) gr.first = s_first, gr.shared = s_shared;

  // ---- the line: work of all items, and of the first window of them
  const int items = a.G + a.B;
  int64_t mine = 0, total = 0;
  for (int i = tid; i < items; i += kThreads) {
    const int64_t x = work_of(a, item_of<D>(a, lens, gr, i));
    if (i < kThreads) mine = x;
    total += x;
  }
#pragma unroll
  for (int o = 32; o; o >>= 1) total += __shfl_xor(total, o);
  if (lane == 0) s_wave[wave] = total;
  __syncthreads();
  total = 0;
  for (int w = 0; w < kWaves; ++w) total += s_wave[w];
  total = uniform(total);
  const int64_t piece = max((total + gridDim.x - 1) / gridDim.x, (int64_t)(row_cost(1) * kWaves * kMinRows));
  const int64_t begin = blockIdx.x * piece, end = min(begin + piece, total);

  int window = 0;     // its first item
  int64_t carry = 0;  // the line before it
  // s_upto[i + 1]: the line up to the window's item i, itself among it
  auto scan = [&]() {
    int64_t sum = mine;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int64_t up = __shfl_up(sum, o);
      if (lane >= o) sum += up;
    }
    __syncthreads();
    if (lane == 63) s_wave[wave] = sum;
    __syncthreads();
    sum += carry;
    for (int w = 0; w < wave; ++w) sum += s_wave[w];
    s_upto[tid + 1] = sum;
    if (tid == 0) s_upto[0] = carry;
    __syncthreads();
  };
  if (begin < end) scan();
  for (int64_t x = begin; x < end;) {
    // ---- the item at x
    while (x >= uniform(s_upto[kThreads])) {
      carry = uniform(s_upto[kThreads]), window += kThreads;
      mine = window + tid < items ? work_of(a, item_of<D>(a, lens, gr, window + tid)) : 0;
      scan();
    }
    __syncthreads();
    if (x < s_upto[tid + 1] && x >= s_upto[tid]) s_item = window + tid, s_start = s_upto[tid];
    __syncthreads();
    const int64_t start = uniform(s_start);
    const int item = uniform(s_item);
    Item it = item_of<D>(a, lens, gr, item);
    it.request = uniform(it.request), it.requests = uniform(it.requests);
    it.lo = uniform(it.lo), it.hi = uniform(it.hi), it.rows = uniform(it.rows);
    it.sets = uniform(it.sets), it.chunks = uniform(it.chunks), it.unit = uniform(it.unit);
    const int cost = row_cost(it.sets), span = it.rows * cost;
    const int u = (int)((x - start) / span);
    const int64_t at = start + (int64_t)u * span;
    const int r0 = (int)((x - at + cost - 1) / cost);
    const int r1 = (int)min((int64_t)it.rows, (end - at + cost - 1) / cost);
    const int kv = u % a.Hkv, chunk = u / a.Hkv;
    const bool own = item >= a.G;
    const int unit = it.unit + u, id = own ? unit - a.group_units : unit;
    if (r0 == 0 && tid == 0) {
      const int from = (int)(at / piece), to = (int)((at + span - cost) / piece);
      a.info[unit] = make_int2(id + from, to - from + 1);
    }
    if (r0 < r1) {
      float* const rec = recs + (own ? a.own_recs + ((int64_t)id + blockIdx.x) * (a.own_cols * (D + 4))
                                     : ((int64_t)id + blockIdx.x) * (16 * max_sets<D>() * (D + 4)));
      if (it.sets == 1)
        walk<D, BF16, 1>(a, in, it, chunk, kv, r0, r1, rec, smem);
      else
        walk<D, BF16, 2>(a, in, it, chunk, kv, r0, r1, rec, smem);
    }
    x = at + span;
  }
}

// Joins the records of a row: a block takes 64 runs of four dims of the rows of one
// (request, KV head), each wave every fourth record.
constexpr int kJoinWaves = 4;
template <int D, bool BF16>
__global__ __launch_bounds__(64 * kJoinWaves) void kv8_shared_join_kernel(
    const float* __restrict__ recs, const int32_t* __restrict__ lens, uint16_t* __restrict__ out,
    float* __restrict__ lse, const Args a, int blocks) {
  constexpr int kPart = D + 4, kAt = 4;
  __shared__ f32x4 s_num[kJoinWaves][64];
  __shared__ f32x2 s_ml[kJoinWaves][64];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int kv = blockIdx.y, b = blockIdx.z, gq = a.Hq / a.Hkv, pairs = gq * a.sq;

  int bad = 0;
  for (int i = tid; i <= a.G; i += 64 * kJoinWaves) {
    const int at = a.first[i];
    bad |= i == 0 ? at != 0 : at < a.first[i - 1];
    if (i == a.G) bad |= at != a.B;
  }
  Groups gr{a.first, a.shared, a.G, true};
  gr.valid = !__syncthreads_or(bad);
  const int group = gr.valid ? gr.of(b) : 0;
  const int shared = gr.valid ? shared_of(a, lens, gr, group) : 0, len = length_of(a, lens, b);

  const int i = blockIdx.x * 64 + lane, pair = min(i / (D / 4), pairs - 1), d4 = i % (D / 4);
  f32x4 num = {0.0f, 0.0f, 0.0f, 0.0f};
  float M = -INFINITY, den = 0.0f;
  auto add = [&](const float* from, int64_t stride, int count) {
    for (int r = wave; r < count; r += kJoinWaves * kAt) {
      f32x4 o[kAt];
      f32x2 ml[kAt];
#pragma unroll
      for (int k = 0; k < kAt; ++k) {
        const float* p = from + min(r + k * kJoinWaves, count - 1) * stride;
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
    const int from = gr.first[group], cols = (gr.first[group + 1] - from) * pairs;
    const int width = 16 * sets_for(D, cols), col = (b - from) * pairs + pair;
    const int unit = (from * pairs / (16 * max_sets<D>()) + group + col / width) * a.Hkv + kv;
    const int2 in = a.info[unit];
    const int64_t stride = (int64_t)(16 * max_sets<D>()) * kPart;
    add(recs + in.x * stride + (int64_t)(col % width) * kPart, stride, min(in.y, blocks));
  }
  if (len > shared) {
    const int width = 16 * sets_for(D, a.own_cols);
    const int unit = (b * a.chunks + pair / width) * a.Hkv + kv;
    const int2 in = a.info[a.group_units + unit];
    const int64_t stride = (int64_t)a.own_cols * kPart;
    add(recs + a.own_recs + in.x * stride + (int64_t)(pair % width) * kPart, stride, min(in.y, blocks));
  }
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

// How the workspace is laid out.
struct Plan {
  int blocks, group_units, chunks, own_cols;
  int64_t own_recs;
  size_t recs, bytes;
};
Plan plan_of(const jf_kv_layout& L, int32_t B, int32_t G, int32_t sq, int32_t Hq) {
  const int D = L.head_dim, Hkv = L.num_kv_heads, pairs = Hq / Hkv * sq;
  const int sets = 2, width = 16 * sets_for(D, pairs);
  Plan p;
  p.blocks = num_cus();
  p.group_units = (int)(((int64_t)B * pairs / (16 * sets) + G + 1) * Hkv);
  p.own_cols = std::min(pairs, width);
  p.chunks = (pairs + width - 1) / width;
  const int64_t own_units = (int64_t)B * p.chunks * Hkv;
  p.own_recs = ((int64_t)p.group_units + p.blocks) * (16 * sets) * (D + 4);
  p.recs = ((size_t)(p.group_units + own_units) * sizeof(int2) + 15) / 16 * 16;
  p.bytes = p.recs + (size_t)(p.own_recs + (own_units + p.blocks) * p.own_cols * (D + 4)) * sizeof(float);
  return p;
}

template <int D, bool BF16>
hipError_t launch_t(const Cache& in, const Args& a, const Plan& p, float* recs, void* out, float* lse,
                    hipStream_t stream) {
  const auto kernel = kv8_shared_kernel<D, BF16>;
  const size_t lds = std::max<size_t>(sizeof(float) * kWaves * 16 * (D + 4), 16 * max_sets<D>() * D * 2);
  if (lds > 49152) {
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel),
                                             hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
    if (e != hipSuccess) return e;
  }
  hipLaunchKernelGGL(kernel, dim3(p.blocks), dim3(kThreads), lds, stream, in.k_codes, in.k_exps,
                     in.v_codes, in.v_exps, in.q, in.tables, in.lens, recs, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int runs = a.Hq / a.Hkv * a.sq * (D / 4);
  hipLaunchKernelGGL((kv8_shared_join_kernel<D, BF16>), dim3((runs + 63) / 64, a.Hkv, a.B),
                     dim3(64 * kJoinWaves), 0, stream, recs, in.lens, static_cast<uint16_t*>(out), lse,
                     a, p.blocks);
  return hipGetLastError();
}

}  // namespace

size_t kv8_shared_bytes(const jf_kv_layout& L, int32_t B, int32_t G, int32_t sq, int32_t Hq) {
  return plan_of(L, B, G, sq, Hq).bytes;
}

hipError_t launch_kv8_shared(const jf_kv_layout& L, const jf_kv_pool_ptrs& pool, bool bf16,
                             const void* q, int32_t B, int32_t sq, int32_t Hq,
                             const int32_t* block_tables, int32_t max_pages, const int32_t* seq_lens,
                             const int32_t* group_start, const int32_t* shared_lens, int32_t G,
                             float softmax_scale, void* ws, void* out, float* lse,
                             hipStream_t stream) {
  const Plan p = plan_of(L, B, G, sq, Hq);
  int shift = 0;
  while ((1 << shift) < L.group_size) ++shift;
  const Cache in{static_cast<const uint8_t*>(pool.k_codes), static_cast<const uint8_t*>(pool.k_meta),
                 static_cast<const uint8_t*>(pool.v_codes), static_cast<const uint8_t*>(pool.v_meta),
                 static_cast<const uint16_t*>(q), block_tables, seq_lens};
  Args a{};
  a.first = group_start, a.shared = shared_lens, a.info = static_cast<int2*>(ws);
  a.B = B, a.G = G, a.sq = sq, a.Hq = Hq, a.Hkv = L.num_kv_heads, a.P = L.page_size;
  a.block_shift = shift, a.num_pages = L.num_pages, a.max_pages = max_pages;
  a.group_units = p.group_units, a.chunks = p.chunks, a.own_cols = p.own_cols, a.own_recs = p.own_recs;
  a.scale_log2 = softmax_scale * 1.44269504088896340736f;
  float* const recs = reinterpret_cast<float*>(static_cast<uint8_t*>(ws) + p.recs);
  auto go = [&](auto fn) { return fn(in, a, p, recs, out, lse, stream); };
  if (L.head_dim == 64) return bf16 ? go(launch_t<64, true>) : go(launch_t<64, false>);
  if (L.head_dim == 128) return bf16 ? go(launch_t<128, true>) : go(launch_t<128, false>);
  return bf16 ? go(launch_t<256, true>) : go(launch_t<256, false>);
}

}  // namespace jfkv
