// Decode attention over the 8-bit cache (format: jfkv_kv8.h): 1-4 causal query
// tokens per request, split over the positions, whose partial results are joined
// by the last block to finish or a second launch, and optionally the attention
// weights of the call added up per position by a second launch.
//
//   s_t = scale * q . k_t,  p_t = exp(s_t - max s),  o = sum p_t v_t / sum p_t
//
// One pass over the pages with a running maximum m and sum l per query (online
// softmax).  The (token, head) pairs that read one KV head are the 16 columns
// of the matrix products (up to 32 pairs: two sets of them for each widened code;
// more: further blocks on the same XCD, which find the pages in its L2):
//   scores  A = K (16 positions x 32 dims), B = Q: lane (n, g) receives column
//           n at positions 4 g .. 4 g + 3;
//   values  A = V (16 dims x 32 positions), B = P: the lane's own eight scores
//           of two tiles, so a probability never leaves its lane.
// Codes enter the matrix cores as fp16 (K beside bf16 queries: bf16), exactly.
// The exponents are one number per tile of 16 positions: K's scales the scores
// (with the softmax scale and log2 e), V's is added to the softmax exponent,
// so P carries 2^(e_v - e_ref) and the accumulators count in units of 2^e_ref.
// e_ref moves (and the accumulators are rescaled) only where e_v - e_ref leaves
// 0 .. 10, and m rises only where a score exceeds it by more than 4 (log2), so
// P stays below 2^14 in fp16.  Scores, m, l and the accumulators are fp32; P is
// rounded to fp16 (2^-11 relative, averaged over the positions).
//
// HBM-bound where it is long: 2 (d + 1 / block) bytes per position and KV head.
// One request of 262,144 positions, 32/8 heads of 128, takes 84 us, 6.4 TB/s; of
// 4,097, 4/1 heads, 8.5 us: a launch, three loads that wait for one another, and
// the join.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "jfkv_internal.h"
#include "jfkv_kv8.h"

namespace jfkv {
namespace {

using namespace kv8;

constexpr int kWaves = 4;
constexpr int kThreads = 64 * kWaves;
constexpr int kRow = 32;       // positions a wave takes at a time (in one page)
constexpr int kCols = 16;      // (token, head) pairs of a block
constexpr int kXcds = 8;

// Splits of a request of L positions.  Rows per wave below which it is not cut
// further: every split costs a start, a merge and a record.  24/4 heads, d = 256,
// 4 / 5 / 6 rows: 4 x 20,000 positions 40 / 36 / 38 us (three tokens 46 / 40 /
// 42), 16 x 4,097 46 / 37 / 39, one request of 4,097 13.9 / 15.3 / 16.5.  32/8
// heads, d = 128, 2 / 3 / 4 rows: 32 x 4,097 72 / 66 / 72, 8 x 9,000 37 / 36 / 37,
// one of 4,097 9.2 / 10.1 / 10.8.
template <int D>
__device__ __forceinline__ int splits_of(int L, int split_cap) {
  constexpr int kMinRows = D > 128 ? 5 : 3;
  const int rows = (L + kRow - 1) / kRow;
  return max(1, min(split_cap, (rows + kWaves * kMinRows - 1) / (kWaves * kMinRows)));
}

template <int D>
struct Row {
  u32x4 k[2][D / 64], v[2][D / 64];
  uint32_t exps;  // lanes 0, 1: K's exponent bytes of the two tiles; 2, 3: V's
};

__device__ __forceinline__ int lane_value(uint32_t x, int l) {
  return __builtin_amdgcn_readlane((int)x, l);
}

// Partial results of some splits: sums of p v and p in units of 2^m.
struct Joined {
  f32x4 num = {0.0f, 0.0f, 0.0f, 0.0f};
  float m = -INFINITY, den = 0.0f;
  __device__ __forceinline__ f32x4 out() const { return num * (den > 0.0f ? 1.0f / den : 0.0f); }
  __device__ __forceinline__ float lse() const { return den > 0.0f ? m + log2f(den) : INFINITY; }
};

// A request's records are joined in one order whichever kernel does it: parts of
// kAt splits by any threads (their loads are in flight together), then the parts
// from the first to the last.
constexpr int kAt = 8;
struct Parts {
  f32x4* num;
  f32x2* ml;
  // m and l of the first `count` of eight records, and the records' factors
  static __device__ __forceinline__ f32x2 weigh(const f32x2 (&r)[kAt], int count, float (&f)[kAt]) {
    float m = r[0].x, den = 0.0f;
#pragma unroll
    for (int k = 1; k < kAt; ++k) m = fmaxf(m, r[k].x);  // (behind count: repeated ones)
#pragma unroll
    for (int k = 0; k < kAt; ++k) {
      f[k] = k >= count || r[k].x == -INFINITY ? 0.0f : exp2_(r[k].x - m);
      den = fmaf(f[k], r[k].y, den);
    }
    return f32x2{m, den};
  }
  // their sums, as part u
  __device__ __forceinline__ void put(int u, const f32x4 (&o)[kAt], const f32x2 (&r)[kAt],
                                      int count) const {
    float f[kAt];
    ml[u] = weigh(r, count, f);
    f32x4 n = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int k = 0; k < kAt; ++k) n += o[k] * f[k];
    num[u] = n;
  }
  // item i of `items` over all parts
  template <bool NUM = true>
  __device__ __forceinline__ Joined get(int i, int items, int parts) const {
    Joined a;
    for (int u = 0; u < parts; ++u) a.m = fmaxf(a.m, ml[u * items + i].x);
    for (int u = 0; u < parts; ++u) {
      const f32x2 r = ml[u * items + i];
      const float f = r.x == -INFINITY ? 0.0f : exp2_(r.x - a.m);
      if (NUM) a.num += num[u * items + i] * f;
      a.den = fmaf(f, r.y, a.den);
    }
    return a;
  }
};
__device__ __forceinline__ Parts parts_at(float* smem, int count) {
  f32x4* const num = reinterpret_cast<f32x4*>(smem);
  return {num, reinterpret_cast<f32x2*>(num + count)};
}
constexpr size_t kPartBytes = sizeof(f32x4) + sizeof(f32x2);

template <int D, bool BF16, bool SUMS, int CS>
__global__ __launch_bounds__(kThreads, D > 128 || CS > 1 ? 2 : 3) void kv8_decode_kernel(
    const uint8_t* __restrict__ k_codes, const uint8_t* __restrict__ k_exps,
    const uint8_t* __restrict__ v_codes, const uint8_t* __restrict__ v_exps,
    const uint16_t* __restrict__ q, const int32_t* __restrict__ block_tables,
    const int32_t* __restrict__ seq_lens, uint32_t* __restrict__ tickets, float* __restrict__ recs,
    float* __restrict__ lse, float* __restrict__ logits, uint16_t* __restrict__ out, int Hq, int sq,
    int Hkv, int P, int block_shift, int num_pages, int max_pages, int max_splits, int split_cap,
    int n_hchunks, bool apart, float scale_log2) {
  constexpr int C = D / 64;
  constexpr int kPart = D + 4;  // floats of a partial: o, m, l (16-byte rows)
  extern __shared__ __align__(16) float smem[];
  const int tid = threadIdx.x, lane = tid & 63, n = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);

  // block -> (split, KV head, column chunk): the chunks of a (split, KV head)
  // on one XCD
  const int slots = split_cap * Hkv;
  const int x8 = blockIdx.x / kXcds;
  const int slot_id = (x8 / n_hchunks) * kXcds + blockIdx.x % kXcds, hc = x8 % n_hchunks;
  if (slot_id >= slots) return;
  const int kv = slot_id % Hkv, split = slot_id / Hkv, b = blockIdx.y;
  const int gq = Hq / Hkv, pairs = gq * sq;
  const int c0 = hc * kCols * CS, ncols = min(kCols * CS, pairs - c0);

  const int L = min(max(seq_lens[b], 0), max_pages * P);
  const int rows = (L + kRow - 1) / kRow, S = splits_of<D>(L, split_cap);
  if (split >= S) return;
  const int base = rows / S, rem = rows % S;
  const int r0 = split * base + min(split, rem), r1 = r0 + base + (split < rem ? 1 : 0);

  // ---- the block's queries as B operands: column n of each set, dims 64 c +
  // 16 g + 8 j ..  In registers, or in LDS where two sets of d = 256 would leave
  // room for one block per CU only (three query tokens of 24/4 heads, 4 x 20,000
  // positions: 61 -> 56 us when that was done).
  constexpr bool kQLds = D > 128 && CS > 1;
  int see[CS];  // positions the columns' queries see
  u32x4 qf[CS][C][2];
  u32x4* const s_q = reinterpret_cast<u32x4*>(smem);
#pragma unroll
  for (int cs = 0; cs < CS; ++cs) {
    const int pair = c0 + min(kCols * cs + n, ncols - 1);  // (columns without a pair repeat the last one)
    const int tok = pair / gq, head = kv * gq + pair % gq;
    see[cs] = L - sq + 1 + tok;
    const uint16_t* qp = q + (((size_t)b * sq + tok) * Hq + head) * D;
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int j = 0; j < 2; ++j)
        if (!kQLds || wave == c % kWaves) {
          const u32x4 x = *reinterpret_cast<const u32x4*>(qp + 64 * c + 16 * g + 8 * j);
          if (kQLds)
            s_q[64 * ((cs * C + c) * 2 + j) + lane] = x;
          else
            qf[cs][c][j] = x;
        }
  }
  if (kQLds) __syncthreads();

  f32x4 acc[CS][C][4] = {};
  float m[CS], l[CS];
#pragma unroll
  for (int cs = 0; cs < CS; ++cs) m[cs] = -INFINITY, l[cs] = 0.0f;
  int e_ref = 0, e_top = -1000;

  // ---- page walk: the wave takes rows r0 + wave, + kWaves, ...  A row's registers
  // are refilled with the next row, K's as soon as the scores are formed and V's
  // after the value products.  Page IDs are read one turn before the loads.
  const int32_t* const table = block_tables + (size_t)b * max_pages;
  const uint32_t koff = n * D + 16 * g, voff = lane * 16;
  const int last = max(r1, 1) - 1;  // (rows past the end read the last one again)
  auto page_of = [&](int r) { return table[min(r, last) * kRow / P]; };
  auto run_of = [&](int pid) {
    return (size_t)((uint32_t)pid < (uint32_t)num_pages ? pid : 0) * Hkv + kv;
  };
  auto fetch_k = [&](Row<D>& w, int r, int pid) {
    const int slot0 = min(r, last) * kRow % P;
    const size_t run = run_of(pid);
    const uint8_t* kp = k_codes + (run * P + slot0) * D;
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int c = 0; c < C; ++c)
        w.k[t][c] = __builtin_nontemporal_load(
            reinterpret_cast<const u32x4*>(kp + koff + t * 16 * D + c * 64));
    const uint8_t* ep = (lane & 2) ? v_exps : k_exps;
    w.exps = ep[run * (P >> block_shift) + ((slot0 + 16 * (lane & 1)) >> block_shift)];
  };
  auto fetch_v = [&](Row<D>& w, int r, int pid) {
    const int slot0 = min(r, last) * kRow % P;
    const uint8_t* vp = v_codes + (run_of(pid) * P + slot0) * D;
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int c = 0; c < C; ++c)
        w.v[t][c] = __builtin_nontemporal_load(
            reinterpret_cast<const u32x4*>(vp + voff + t * 16 * D + c * 1024));
  };

  // a row's scores to the workspace, for the sums of the weights
  auto keep_scores = [&](int r, const float (&s)[CS][2][4]) {
#pragma unroll
    for (int cs = 0; cs < CS; ++cs)
      if (kCols * cs + n < ncols) {
        float* const lg = logits + (((size_t)b * Hkv + kv) * pairs + c0 + kCols * cs + n) *
                                       ((size_t)max_pages * P) + r * kRow + 4 * g;
#pragma unroll
        for (int t = 0; t < 2; ++t)
          *reinterpret_cast<f32x4*>(lg + 16 * t) =
              f32x4{s[cs][t][0], s[cs][t][1], s[cs][t][2], s[cs][t][3]};
      }
  };
  // scores of a row in log2 units, and the exponents of its values
  auto scores = [&](const Row<D>& w, int r, float (&s)[CS][2][4], int (&ev)[2]) {
    const int pos0 = r * kRow;
    f32x4 a[2][CS] = {};
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
          for (int cs = 0; cs < CS; ++cs) a[t][cs] = mma<BF16>(k, qc[cs], a[t][cs]);
        }
      }
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const float f = scale_log2 * power2(lane_value(w.exps, t) - 127);
      ev[t] = lane_value(w.exps, 2 + t) - 127;
#pragma unroll
      for (int cs = 0; cs < CS; ++cs)
#pragma unroll
        for (int i = 0; i < 4; ++i) s[cs][t][i] = a[t][cs][i] * f;
    }
    if (pos0 + kRow > L - sq + 1) {
      // positions that a query does not see, and slots not written yet (their codes,
      // a NaN among them, and exponents are not looked at)
#pragma unroll
      for (int cs = 0; cs < CS; ++cs)
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (pos0 + 16 * t + 4 * g + i >= see[cs]) s[cs][t][i] = -INFINITY;
      if (pos0 + 16 >= L) ev[1] = ev[0];
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
    if (pos0 + kRow > L) {  // slots not written yet: zeros (their codes may be NaN)
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const int a = min(max(L - pos0 - 16 * t - 4 * g, 0), 4);
        const uint32_t keep = a ? 0xffffffffu >> (8 * (4 - a)) : 0u;
#pragma unroll
        for (int c = 0; c < C; ++c) w.v[t][c] &= keep;
      }
    }
    // both tiles with one reference, or one after the other where their exponents
    // are too far apart for that
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
          // (opaque: widened ahead of the loop over the parts, all operands would
          // be held at once)
          uint32_t v0 = w.v[0][c][dt], v1 = w.v[1][c][dt];
          asm volatile("" : "+v"(v0), "+v"(v1));
          const u32x4 a = widen8<false>(v0, v1);
#pragma unroll
          for (int cs = 0; cs < CS; ++cs) acc[cs][c][dt] = mma<false>(a, pf[cs], acc[cs][c][dt]);
        }
    }
  };

  if (r0 < r1) {
    // One row in flight: four waves then keep 32 KB (at d = 128) on the way per CU,
    // and three blocks fit on one; two took 86.9 against 85.2 us at 262,144 positions
    // and 80 against 70 for eight requests of 20,000.
    Row<D> w;
    int r = r0 + wave;
    int pid = page_of(r), ahead = page_of(r + kWaves);
    fetch_k(w, r, pid);
    fetch_v(w, r, pid);
    for (; r < r1; r += kWaves) {
      const bool on = (uint32_t)pid < (uint32_t)num_pages;
      float s[CS][2][4];
      int ev[2];
      scores(w, r, s, ev);
      if (!on) {
#pragma unroll
        for (int cs = 0; cs < CS; ++cs)
#pragma unroll
          for (int e = 0; e < 8; ++e) s[cs][e / 4][e % 4] = -INFINITY;
      }
      if (SUMS) keep_scores(r, s);
      fetch_k(w, r + kWaves, ahead);
      if (on) attend(w, r, s, ev);
      fetch_v(w, r + kWaves, ahead);
      pid = ahead;
      ahead = page_of(r + 2 * kWaves);
    }
  }

  const size_t rec0 = ((size_t)b * Hkv + kv) * pairs + c0;  // the block's first (request, pair)
  // the block's records, written and read with device-scope coherent accesses
  const __amdgpu_buffer_rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc(
      recs + rec0 * max_splits * kPart, (short)0, (int)(ncols * max_splits * kPart * 4), 0x00020000);
  constexpr int kSc1 = 16;
  auto store_rec = [&](int col, int d4, f32x4 o, float M, float den) {
    const int rec = (col * max_splits + split) * kPart * 4;
    __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, o), rs, rec + 16 * d4, 0, kSc1);
    if (d4 == 0)
      __builtin_amdgcn_raw_buffer_store_b64(
          __builtin_bit_cast(u32x2, f32x2{M, den}), rs, rec + 4 * D, 0, kSc1);
  };
  auto store_out = [&](int col, int d4, f32x4 o) {
    const int pr = c0 + col;
    uint16_t* op = out + (((size_t)b * sq + pr / gq) * Hq + kv * gq + pr % gq) * D + 4 * d4;
    *reinterpret_cast<uint2*>(op) = make_uint2(narrow2<BF16>(o.x, o.y), narrow2<BF16>(o.z, o.w));
  };
  // ---- merge the waves in LDS, one set of columns after the other: o (units 1),
  // m, l
  const int wide = min(kCols, ncols) * kPart;  // floats of a wave
#pragma unroll
  for (int cs = 0; cs < CS; ++cs) {
    const int here = min(kCols, ncols - kCols * cs);  // columns of the set
    const float den = col_sum(l[cs]);
    float* const mine = smem + wave * wide + n * kPart;
    if (kQLds || cs) __syncthreads();  // (LDS still held the queries or the last set)
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
      const int at = i / (D / 4), col = kCols * cs + at, d4 = i % (D / 4);
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
      if (S == 1) {
        store_out(col, d4, num * (sum > 0.0f ? 1.0f / sum : 0.0f));
        if (SUMS && d4 == 0) lse[rec0 + col] = sum > 0.0f ? M + log2f(sum) : INFINITY;
      } else {
        store_rec(col, d4, num, M, sum);
      }
    }
  }
  if (S == 1 || apart) return;

  // ---- the last split to finish combines the records.  Every word the blocks exchange is written
  // and read by device-scope coherent accesses (sc1: written through to, and read
  // from, the level that all XCDs share); each thread waits for its
  // record stores before the barrier that precedes the ticket, and the combining
  // block loads records only after it has seen the last ticket (the decode over
  // 4-bit pages argues this exchange in full).
  uint32_t* const s_ticket = reinterpret_cast<uint32_t*>(smem);
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
  if (tid == 0) {
    uint32_t* const ticket = tickets + ((size_t)b * Hkv + kv) * n_hchunks + hc;
    const uint32_t t = __hip_atomic_fetch_add(ticket, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    if (t == (uint32_t)(S - 1))
      __hip_atomic_store(ticket, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    *s_ticket = t;
  }
  __syncthreads();
  if (*s_ticket != (uint32_t)(S - 1)) return;
  const int items = ncols * (D / 4), parts = (S + kAt - 1) / kAt;
  const Parts at = parts_at(smem + 4, items * parts);
  for (int u = tid; u < items * parts; u += kThreads) {
    const int i = u % items, col = i / (D / 4), s0 = u / items * kAt;
    f32x4 o[kAt];
    f32x2 ml[kAt];
#pragma unroll
    for (int k = 0; k < kAt; ++k) {
      const int rec = (col * max_splits + min(s0 + k, S - 1)) * kPart * 4;
      o[k] = __builtin_bit_cast(
          f32x4, __builtin_amdgcn_raw_buffer_load_b128(rs, rec + 16 * (i % (D / 4)), 0, kSc1));
      ml[k] = __builtin_bit_cast(f32x2, __builtin_amdgcn_raw_buffer_load_b64(rs, rec + 4 * D, 0, kSc1));
    }
    at.put(u, o, ml, S - s0);
  }
  __syncthreads();
  for (int i = tid; i < items; i += kThreads) {
    const Joined sum = at.get(i, items, parts);
    store_out(i / (D / 4), i % (D / 4), sum.out());
    if (SUMS && i % (D / 4) == 0) lse[rec0 + i / (D / 4)] = sum.lse();
  }
}

// Adds the weights exp2(s_t - z) of pairs p0 .. p0 + n - 1 (scores lg [pair][cap], z
// from zs) at four positions.
__device__ __forceinline__ void add_pairs(f32x4& sum, const float* lg, size_t cap, const float* zs,
                                          int n) {
  constexpr int kAhead = 6;  // loads on the way (one: 9.1 us for 6.1 of 78,000 positions, 18 pairs)
  for (int i0 = 0; i0 < n; i0 += kAhead) {
    f32x4 s[kAhead];
    float z[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      const int i = min(i0 + k, n - 1);
      s[k] = *reinterpret_cast<const f32x4*>(lg + (size_t)i * cap);
      z[k] = i0 + k < n ? zs[i] : INFINITY;
    }
#pragma unroll
    for (int k = 0; k < kAhead; ++k)
#pragma unroll
      for (int e = 0; e < 4; ++e) sum[e] += exp2_(s[k][e] - z[k]);
  }
}
__device__ __forceinline__ void store_sums(float* w, int64_t t, int L, const f32x4& sum) {
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (t + e < L) w[t + e] += sum[e];
}

// The same where a launch of its own joins the records: a workgroup per (request,
// KV head, pair).  SUMS: and workgroups behind them for the weights' sums, 1,024
// positions each, which take the log-sum-exps from the records themselves rather
// than wait for another launch.
template <int D, bool BF16, bool SUMS>
__global__ __launch_bounds__(kThreads) void kv8_join_kernel(
    const float* __restrict__ recs, const int32_t* __restrict__ seq_lens,
    const float* __restrict__ lse, uint16_t* __restrict__ out, const float* __restrict__ logits,
    float* __restrict__ weights, int64_t stride, int pairs, int Hq, int sq, int cap, int max_splits,
    int split_cap) {
  constexpr int kPer = D / 4;
  extern __shared__ __align__(16) float smem[];
  const int pair = blockIdx.x, kv = blockIdx.y, b = blockIdx.z, Hkv = gridDim.y;
  const int L = min(max(seq_lens[b], 0), cap), S = splits_of<D>(L, split_cap);
  const int tid = threadIdx.x, parts = (S + kAt - 1) / kAt;
  const size_t row = (size_t)b * Hkv + kv;
  const Parts at = parts_at(smem, kPer * parts);
  if (SUMS && pair >= pairs) {
    constexpr int kChunk = 32;  // pairs at a time
    f32x2* const ml = reinterpret_cast<f32x2*>(smem);        // [part][pair]
    float* const zs = reinterpret_cast<float*>(ml + kChunk * parts);
    const int64_t t0 = (int64_t)(pair - pairs) * (4 * kThreads), t = t0 + 4 * tid;
    if (t0 >= L) return;
    f32x4 sum = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int p0 = 0; p0 < pairs; p0 += kChunk) {
      const int n = min(kChunk, pairs - p0);
      if (S == 1) {
        if (tid < n) zs[tid] = lse[row * pairs + p0 + tid];
      } else {
        for (int u = tid; u < n * parts; u += kThreads) {
          const int s0 = u / n * kAt;
          const float* const from = recs + (row * pairs + p0 + u % n) * max_splits * (D + 4) + D;
          f32x2 r[kAt];
          float f[kAt];
#pragma unroll
          for (int k = 0; k < kAt; ++k)
            r[k] = *reinterpret_cast<const f32x2*>(from + (size_t)min(s0 + k, S - 1) * (D + 4));
          ml[u] = Parts::weigh(r, S - s0, f);
        }
        __syncthreads();
        if (tid < n) zs[tid] = Parts{nullptr, ml}.template get<false>(tid, n, parts).lse();
      }
      __syncthreads();
      if (t < L) add_pairs(sum, logits + (row * pairs + p0) * (size_t)cap + t, cap, zs, n);
      __syncthreads();
    }
    store_sums(weights + row * stride, t, L, sum);
    return;
  }
  if (S == 1) return;  // (the output is there)
  const float* const from = recs + (row * pairs + pair) * max_splits * (D + 4);
  for (int u = tid; u < kPer * parts; u += kThreads) {
    const int s0 = u / kPer * kAt;
    f32x4 o[kAt];
    f32x2 ml[kAt];
#pragma unroll
    for (int k = 0; k < kAt; ++k) {
      const float* p = from + (size_t)min(s0 + k, S - 1) * (D + 4);
      o[k] = *reinterpret_cast<const f32x4*>(p + 4 * (u % kPer));
      ml[k] = *reinterpret_cast<const f32x2*>(p + D);
    }
    at.put(u, o, ml, S - s0);
  }
  __syncthreads();
  if (tid >= kPer) return;
  const int gq = Hq / Hkv;
  const f32x4 r = at.get(tid, kPer, parts).out();
  uint16_t* op = out + (((size_t)b * sq + pair / gq) * Hq + kv * gq + pair % gq) * D + 4 * tid;
  *reinterpret_cast<uint2*>(op) = make_uint2(narrow2<BF16>(r.x, r.y), narrow2<BF16>(r.z, r.w));
}

// weights[b][kv][t] += sum over the pairs of exp2(s_t - lse) where the decode itself
// left the log-sum-exps of its pairs (and the scores, log2 units).  Four positions
// per thread; positions from the request's length on are left as they are.
__global__ __launch_bounds__(kThreads) void kv8_sums_kernel(const float* __restrict__ logits,
                                                            const float* __restrict__ lse,
                                                            const int32_t* __restrict__ seq_lens,
                                                            float* __restrict__ weights,
                                                            int64_t stride, int pairs, int cap) {
  const int b = blockIdx.z, kv = blockIdx.y, Hkv = gridDim.y;
  const int L = min(max(seq_lens[b], 0), cap);
  const int64_t t = ((int64_t)blockIdx.x * kThreads + threadIdx.x) * 4;
  if (t >= L) return;
  const size_t row = (size_t)b * Hkv + kv;
  f32x4 sum = {0.0f, 0.0f, 0.0f, 0.0f};
  add_pairs(sum, logits + row * pairs * (size_t)cap + t, cap, lse + row * pairs, pairs);
  store_sums(weights + row * stride, t, L, sum);
}

template <int D, bool BF16, bool SUMS, int CS>
hipError_t launch_cs(const jf_kv_layout& L, const jf_kv_pool_ptrs& pool, const void* q, int32_t B,
                  int32_t sq, int32_t Hq, const int32_t* bt, int32_t max_pages, const int32_t* lens,
                  float scale, int32_t max_splits, void* ws, void* out, float* weights,
                  int64_t stride, hipStream_t stream) {
  const int Hkv = L.num_kv_heads, pairs = Hq / Hkv * sq;
  const int n_hchunks = (pairs + kCols * CS - 1) / (kCols * CS);
  // enough blocks for one per CU when one request runs alone; the count
  // depends on neither the batch nor the lengths, so that a request's output
  // is bitwise the same in any batch
  const int split_cap = (int)std::max<int64_t>(
      1, std::min<int64_t>(max_splits, num_cus() / ((int64_t)Hkv * n_hchunks)));
  const int64_t slots = ((int64_t)split_cap * Hkv + kXcds - 1) / kXcds * kXcds;
  // A unit's records are joined by the last of its blocks, which saves a launch,
  // or by a launch of its own, a block per pair, where one CU would read them for
  // too long.  In the kernel / apart: one request of 4,097 positions, 4/1 heads,
  // d = 128 (128 KB) 8.5 / 8.8 us, 16/8 heads of 64 8.0 / 8.7; four of 35,000 15.8 /
  // 12.8; one of 30,000, 24/4 heads, d = 256 (384 KB) 24.5 / 19.1, three tokens
  // (1.1 MB) 38.3 / 21.9.
  const int64_t items = (int64_t)std::min(kCols * CS, pairs) * (D / 4);
  const int parts = (split_cap + kAt - 1) / kAt;
  const bool apart = B > 1 || items * 16 * split_cap > 131072;
  const Kv8Workspace at = kv8_workspace(B, sq, Hq, D, max_splits, SUMS ? max_pages * L.page_size : 0);
  uint8_t* base = static_cast<uint8_t*>(ws);
  float* lse = reinterpret_cast<float*>(base + at.lse);
  float* logits = reinterpret_cast<float*>(base + at.logits);
  int shift = 0;
  while ((1 << shift) < L.group_size) ++shift;
  // the waves' partials; then the ticket and the records' parts
  const size_t lds = std::max<size_t>(sizeof(float) * kWaves * std::min(kCols, pairs) * (D + 4),
                                      16 + (apart ? 0 : items * parts * kPartBytes));
  const auto kernel = kv8_decode_kernel<D, BF16, SUMS, CS>;
  if (lds > 65536) {
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel),
                                             hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
    if (e != hipSuccess) return e;
  }
  hipLaunchKernelGGL(kernel, dim3((uint32_t)(slots * n_hchunks), B), dim3(kThreads), lds, stream,
                     static_cast<const uint8_t*>(pool.k_codes),
                     static_cast<const uint8_t*>(pool.k_meta),
                     static_cast<const uint8_t*>(pool.v_codes),
                     static_cast<const uint8_t*>(pool.v_meta), static_cast<const uint16_t*>(q), bt,
                     lens, reinterpret_cast<uint32_t*>(base),
                     reinterpret_cast<float*>(base + at.records), lse, logits,
                     static_cast<uint16_t*>(out), Hq, sq, Hkv, L.page_size, shift, L.num_pages,
                     max_pages, max_splits, split_cap, n_hchunks, apart, scale * 1.44269504088896340736f);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int cap = max_pages * L.page_size, sums = (cap + 4 * kThreads - 1) / (4 * kThreads);
  if (apart && split_cap > 1) {
    hipLaunchKernelGGL((kv8_join_kernel<D, BF16, SUMS>), dim3(pairs + (SUMS ? sums : 0), Hkv, B),
                       dim3(kThreads), D / 4 * parts * kPartBytes, stream,
                       reinterpret_cast<const float*>(base + at.records), lens, lse,
                       static_cast<uint16_t*>(out), logits, weights, stride, pairs, Hq, sq, cap,
                       max_splits, split_cap);
  } else if (SUMS) {
    hipLaunchKernelGGL(kv8_sums_kernel, dim3(sums, Hkv, B), dim3(kThreads), 0, stream, logits, lse,
                       lens, weights, stride, pairs, cap);
  }
  return hipGetLastError();
}

template <int D, bool BF16, bool SUMS>
hipError_t launch(const jf_kv_layout& L, const jf_kv_pool_ptrs& pool, const void* q, int32_t B,
                  int32_t sq, int32_t Hq, const int32_t* bt, int32_t max_pages, const int32_t* lens,
                  float scale, int32_t max_splits, void* ws, void* out, float* weights,
                  int64_t stride, hipStream_t stream) {
  const auto go = Hq / L.num_kv_heads * sq > kCols ? launch_cs<D, BF16, SUMS, 2>
                                                   : launch_cs<D, BF16, SUMS, 1>;
  return go(L, pool, q, B, sq, Hq, bt, max_pages, lens, scale, max_splits, ws, out, weights, stride,
            stream);
}

}  // namespace

hipError_t launch_kv8_decode(const jf_kv_layout& L, const jf_kv_pool_ptrs& pool, bool bf16,
                             const void* q, int32_t B, int32_t sq, int32_t Hq,
                             const int32_t* block_tables, int32_t max_pages,
                             const int32_t* seq_lens, float softmax_scale, int32_t max_splits,
                             void* ws, void* out, float* weights, int64_t stride,
                             hipStream_t stream) {
  auto go = [&](auto fn) {
    return fn(L, pool, q, B, sq, Hq, block_tables, max_pages, seq_lens, softmax_scale, max_splits,
              ws, out, weights, stride, stream);
  };
#define JF_CASE(D_)                                                              \
  if (L.head_dim == D_) {                                                        \
    if (weights) return bf16 ? go(launch<D_, true, true>) : go(launch<D_, false, true>); \
    return bf16 ? go(launch<D_, true, false>) : go(launch<D_, false, false>);    \
  }
  JF_CASE(64)
  JF_CASE(128)
  JF_CASE(256)
#undef JF_CASE
  return hipErrorInvalidValue;
}

}  // namespace jfkv
