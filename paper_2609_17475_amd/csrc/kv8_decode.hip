// Decode attention over the 8-bit cache (format: jfkv_kv8.h): 1-4 causal query
// tokens per request, split over the positions, with an in-kernel combine, and
// optionally the attention weights of the call added up per position.
//
//   s_t = scale * q . k_t,  p_t = exp(s_t - max s),  o = sum p_t v_t / sum p_t
//
// One pass over the pages with a running maximum m and sum l per query (online
// softmax).  The (token, head) pairs that read one KV head are the 16 columns
// of the matrix products (more pairs: further blocks on the same XCD, which
// find the pages in its L2):
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
// HBM-bound: 2 (d + 1 / block) bytes per position and KV head.
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
constexpr int kCols = 16;      // (token, head) pairs of a block
constexpr int kXcds = 8;
constexpr float kMargin = 4.0f;  // m is raised where a score exceeds it by more (log2)
constexpr int kRefMax = 10;      // e_v - e_ref stays in 0 .. kRefMax
constexpr int kRefFloor = 80;    // e_ref is not lowered further than this below the largest e_v

template <int D>
struct Row {
  u32x4 k[2][D / 64], v[2][D / 64];
  uint32_t exps;  // lanes 0, 1: K's exponent bytes of the two tiles; 2, 3: V's
};

__device__ __forceinline__ float exp2_(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ int lane_value(uint32_t x, int l) {
  return __builtin_amdgcn_readlane((int)x, l);
}

// The maximum (sum) over the four lanes that hold a column.
__device__ __forceinline__ float col_max(float x) {
  x = fmaxf(x, __shfl_xor(x, 16));
  return fmaxf(x, __shfl_xor(x, 32));
}
__device__ __forceinline__ float col_sum(float x) {
  x += __shfl_xor(x, 16);
  return x + __shfl_xor(x, 32);
}

template <int D, bool BF16, bool SUMS>
__global__ __launch_bounds__(kThreads) void kv8_decode_kernel(
    const uint8_t* __restrict__ k_codes, const uint8_t* __restrict__ k_exps,
    const uint8_t* __restrict__ v_codes, const uint8_t* __restrict__ v_exps,
    const uint16_t* __restrict__ q, const int32_t* __restrict__ block_tables,
    const int32_t* __restrict__ seq_lens, uint32_t* __restrict__ tickets, float* __restrict__ recs,
    float* __restrict__ lse, float* __restrict__ logits, uint16_t* __restrict__ out, int Hq, int sq,
    int Hkv, int P, int block_shift, int num_pages, int max_pages, int max_splits, int split_cap,
    int n_hchunks, float scale_log2) {
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
  const int c0 = hc * kCols, ncols = min(kCols, pairs - c0);

  const int L = min(max(seq_lens[b], 0), max_pages * P);
  const int rows = (L + kRow - 1) / kRow;
  const int S = max(1, min(split_cap, (rows + kWaves - 1) / kWaves));
  if (split >= S) return;
  const int base = rows / S, rem = rows % S;
  const int r0 = split * base + min(split, rem), r1 = r0 + base + (split < rem ? 1 : 0);

  // ---- the block's queries as B operands: column n, dims 64 c + 16 g + 8 j ..
  const int pair = c0 + min(n, ncols - 1);  // (columns without a pair repeat the last one)
  const int tok = pair / gq, head = kv * gq + pair % gq;
  const int see = L - sq + 1 + tok;  // positions the column's query sees
  u32x4 qf[C][2];
  {
    const uint16_t* qp = q + (((size_t)b * sq + tok) * Hq + head) * D;
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int j = 0; j < 2; ++j)
        qf[c][j] = *reinterpret_cast<const u32x4*>(qp + 64 * c + 16 * g + 8 * j);
  }

  f32x4 acc[C][4] = {};
  float m = -INFINITY, l = 0.0f;
  int e_ref = 0, e_top = -1000;

  // ---- page walk: the wave takes rows r0 + wave, + kWaves, ...  NB rows are in
  // flight: a row's registers are refilled with the row NB turns ahead, K's as
  // soon as the scores are formed and V's after the value products.  Page IDs
  // are read one turn before the loads that need them.
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

  // scores of a row in log2 units, and the exponents of its values
  auto scores = [&](const Row<D>& w, int r, bool on, float (&s)[2][4], int (&ev)[2]) {
    const int pos0 = r * kRow;
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      f32x4 a = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int c = 0; c < C; ++c) {
        a = mma<BF16>(widen8<BF16>(w.k[t][c].x, w.k[t][c].y), qf[c][0], a);
        a = mma<BF16>(widen8<BF16>(w.k[t][c].z, w.k[t][c].w), qf[c][1], a);
      }
      const float f = scale_log2 * power2(lane_value(w.exps, t) - 127);
      ev[t] = lane_value(w.exps, 2 + t) - 127;
#pragma unroll
      for (int i = 0; i < 4; ++i) s[t][i] = a[i] * f;
    }
    if (!on || pos0 + kRow > L - sq + 1) {
      // positions that a query does not see, slots not written yet (their codes,
      // a NaN among them, and exponents are not looked at), pages outside the pool
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (!on || pos0 + 16 * t + 4 * g + i >= see) s[t][i] = -INFINITY;
      if (pos0 + 16 >= L) ev[1] = ev[0];
    }
    if constexpr (SUMS)
      if (n < ncols) {
        float* const lg = logits + (((size_t)b * Hkv + kv) * pairs + c0 + n) *
                                       ((size_t)max_pages * P) + pos0 + 4 * g;
        *reinterpret_cast<f32x4*>(lg) = f32x4{s[0][0], s[0][1], s[0][2], s[0][3]};
        *reinterpret_cast<f32x4*>(lg + 16) = f32x4{s[1][0], s[1][1], s[1][2], s[1][3]};
      }
  };
  auto rescale = [&](float f) {
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int dt = 0; dt < 4; ++dt) acc[c][dt] *= f;
  };
  // e_ref such that lo .. hi lie in its window
  auto refer = [&](int lo, int hi) {
    e_top = max(e_top, hi);
    if (lo >= e_ref && hi <= e_ref + kRefMax) return;
    const int e = max(max(hi - kRefMax, lo - 4), e_top - kRefFloor);
    rescale(__builtin_ldexpf(1.0f, e_ref - e));
    e_ref = e;
  };
  // P of a tile in units of 2^(e_ref - ev), its sum into l
  auto weigh = [&](const float (&s)[4], float mu, int ev, uint32_t (&pf)[2]) {
    const float by = (float)(ev - e_ref);
    float p[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) p[i] = exp2_(s[i] - mu + by);
    if (ev - e_ref >= -kRefMax) {
      l = fmaf((p[0] + p[1]) + (p[2] + p[3]), power2(e_ref - ev), l);
    } else {  // (far below the largest values: P may vanish, l must not)
      for (int i = 0; i < 4; ++i) l += exp2_(s[i] - mu);
    }
    pf[0] = narrow2<false>(p[0], p[1]), pf[1] = narrow2<false>(p[2], p[3]);
  };
  auto values = [&](const Row<D>& w, u32x4 pf, uint32_t keep0, uint32_t keep1) {
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int dt = 0; dt < 4; ++dt)
        acc[c][dt] = mma<false>(widen8<false>(w.v[0][c][dt] & keep0, w.v[1][c][dt] & keep1), pf,
                                acc[c][dt]);
  };
  auto attend = [&](const Row<D>& w, int r, const float (&s)[2][4], const int (&ev)[2]) {
    const int pos0 = r * kRow;
    float top = fmaxf(fmaxf(s[0][0], s[0][1]), fmaxf(s[0][2], s[0][3]));
    top = fmaxf(top, fmaxf(fmaxf(s[1][0], s[1][1]), fmaxf(s[1][2], s[1][3])));
    if (__any(top > m + kMargin)) {
      const float mn = fmaxf(m, col_max(top));
      const float f = m == -INFINITY ? 0.0f : exp2_(m - mn);
      l *= f;
      rescale(f);
      m = mn;
    }
    const float mu = m == -INFINITY ? 0.0f : m;
    uint32_t keep0 = 0xffffffffu, keep1 = 0xffffffffu;
    if (pos0 + kRow > L) {
      const int a = min(max(L - pos0 - 4 * g, 0), 4), c = min(max(L - pos0 - 16 - 4 * g, 0), 4);
      keep0 = a ? 0xffffffffu >> (8 * (4 - a)) : 0u;
      keep1 = c ? 0xffffffffu >> (8 * (4 - c)) : 0u;
    }
    const int lo = min(ev[0], ev[1]), hi = max(ev[0], ev[1]);
    uint32_t p0[2], p1[2];
    if (hi - lo <= kRefMax) {
      refer(lo, hi);
      weigh(s[0], mu, ev[0], p0);
      weigh(s[1], mu, ev[1], p1);
      values(w, u32x4{p0[0], p0[1], p1[0], p1[1]}, keep0, keep1);
    } else {  // too far apart for one reference: tile by tile
      refer(ev[0], ev[0]);
      weigh(s[0], mu, ev[0], p0);
      values(w, u32x4{p0[0], p0[1], 0u, 0u}, keep0, 0u);
      refer(ev[1], ev[1]);
      weigh(s[1], mu, ev[1], p1);
      values(w, u32x4{0u, 0u, p1[0], p1[1]}, 0u, keep1);
    }
  };

  if (r0 < r1) {
    constexpr int NB = D > 128 ? 1 : 2;
    Row<D> w[NB];
    int pid[NB], ahead[NB];
#pragma unroll
    for (int i = 0; i < NB; ++i) {
      const int r = r0 + wave + i * kWaves;
      pid[i] = page_of(r);
      ahead[i] = page_of(r + NB * kWaves);
      fetch_k(w[i], r, pid[i]);
      fetch_v(w[i], r, pid[i]);
    }
    for (int rr = r0 + wave; rr < r1; rr += NB * kWaves) {
#pragma unroll
      for (int i = 0; i < NB; ++i) {
        const int r = rr + i * kWaves, rn = r + NB * kWaves;
        const bool on = (uint32_t)pid[i] < (uint32_t)num_pages;
        float s[2][4];
        int ev[2];
        if (r < r1) scores(w[i], r, on, s, ev);
        fetch_k(w[i], rn, ahead[i]);
        if (r < r1 && on) attend(w[i], r, s, ev);
        fetch_v(w[i], rn, ahead[i]);
        pid[i] = ahead[i];
        ahead[i] = page_of(rn + NB * kWaves);
      }
    }
  }

  // ---- merge the waves in LDS: o (units 1), m, l of the block's columns
  l = col_sum(l);
  {
    float* part = smem + (size_t)(wave * ncols + n) * kPart;
    if (n < ncols) {
      const float f = __builtin_ldexpf(1.0f, e_ref);
#pragma unroll
      for (int c = 0; c < C; ++c)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          *reinterpret_cast<f32x4*>(part + 64 * c + 16 * g + 4 * i) =
              f32x4{acc[c][0][i], acc[c][1][i], acc[c][2][i], acc[c][3][i]} * f;
      if (g == 0) part[D] = m, part[D + 1] = l;
    }
  }
  __syncthreads();
  const size_t rec0 = ((size_t)b * Hkv + kv) * pairs + c0;  // the block's first (request, pair)
  auto store_out = [&](int col, int d4, f32x4 o) {
    const int pr = c0 + col;
    uint16_t* op = out + (((size_t)b * sq + pr / gq) * Hq + kv * gq + pr % gq) * D + 4 * d4;
    *reinterpret_cast<uint2*>(op) = make_uint2(narrow2<BF16>(o.x, o.y), narrow2<BF16>(o.z, o.w));
  };
  for (int i = tid; i < ncols * (D / 4); i += kThreads) {
    const int col = i / (D / 4), d4 = i % (D / 4);
    float mw[kWaves], M = -INFINITY, den = 0.0f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      mw[w] = smem[(size_t)(w * ncols + col) * kPart + D];
      M = fmaxf(M, mw[w]);
    }
    f32x4 num = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const float* part = smem + (size_t)(w * ncols + col) * kPart;
      const float f = mw[w] == -INFINITY ? 0.0f : exp2_(mw[w] - M);
      num += *reinterpret_cast<const f32x4*>(part + 4 * d4) * f;
      den = fmaf(f, part[D + 1], den);
    }
    if (S == 1) {
      store_out(col, d4, num * (den > 0.0f ? 1.0f / den : 0.0f));
      if (SUMS && d4 == 0) lse[rec0 + col] = den > 0.0f ? M + log2f(den) : INFINITY;
    } else {
      // agent-scope stores: written through to the device-coherent level, where
      // the block that combines (on any XCD) reads them
      float* rec = recs + ((rec0 + col) * max_splits + split) * kPart;
#pragma unroll
      for (int e = 0; e < 4; ++e)
        __hip_atomic_store(rec + 4 * d4 + e, num[e], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      if (d4 == 0) {
        __hip_atomic_store(rec + D, M, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        __hip_atomic_store(rec + D + 1, den, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      }
    }
  }
  if (S == 1) return;

  // ---- the last split to finish combines the records.  Every word the blocks
  // exchange is written and read by device-scope atomic instructions; each
  // thread waits for its record stores before the barrier that precedes the
  // ticket, and the combining block loads records only after it has seen the
  // last ticket (the decode over 4-bit pages argues this exchange in full).
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
  uint32_t* const ticket = tickets + ((size_t)b * Hkv + kv) * n_hchunks + hc;
  uint32_t* const s_ticket = reinterpret_cast<uint32_t*>(smem);
  if (tid == 0)
    *s_ticket = __hip_atomic_fetch_add(ticket, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  __syncthreads();
  if (*s_ticket != (uint32_t)(S - 1)) return;
  if (tid == 0) __hip_atomic_store(ticket, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  auto load = [&](const float* p) {
    return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  };
  for (int i = tid; i < ncols * (D / 4); i += kThreads) {
    const int col = i / (D / 4), d4 = i % (D / 4);
    const float* rec = recs + (rec0 + col) * max_splits * kPart;
    float M = -INFINITY, den = 0.0f;
    f32x4 num = {0.0f, 0.0f, 0.0f, 0.0f};
    constexpr int kAt = 8;  // records in flight
    for (int s0 = 0; s0 < S; s0 += kAt) {
      f32x4 o[kAt];
      float ms[kAt], ls[kAt];
#pragma unroll
      for (int k = 0; k < kAt; ++k) {
        const float* rs = rec + (size_t)min(s0 + k, S - 1) * kPart;
#pragma unroll
        for (int e = 0; e < 4; ++e) o[k][e] = load(rs + 4 * d4 + e);
        ms[k] = load(rs + D), ls[k] = load(rs + D + 1);
      }
      float mx = M;
#pragma unroll
      for (int k = 0; k < kAt; ++k) {
        if (s0 + k >= S) ms[k] = -INFINITY;
        mx = fmaxf(mx, ms[k]);
      }
      const float f = M == -INFINITY ? 0.0f : exp2_(M - mx);
      num *= f, den *= f, M = mx;
#pragma unroll
      for (int k = 0; k < kAt; ++k) {
        const float fk = ms[k] == -INFINITY ? 0.0f : exp2_(ms[k] - M);
        num += o[k] * fk;
        den = fmaf(fk, ls[k], den);
      }
    }
    store_out(col, d4, num * (den > 0.0f ? 1.0f / den : 0.0f));
    if (SUMS && d4 == 0) lse[rec0 + col] = den > 0.0f ? M + log2f(den) : INFINITY;
  }
}

// weights[b][kv][t] += sum over the pairs of exp2(s_t - lse): the decode left
// the scores (log2 units) and the log-sum-exps of its pairs.  Four positions
// per thread; positions from the request's length on are left as they are.
__global__ __launch_bounds__(256) void kv8_sums_kernel(const float* __restrict__ logits,
                                                       const float* __restrict__ lse,
                                                       const int32_t* __restrict__ seq_lens,
                                                       float* __restrict__ weights, int64_t stride,
                                                       int pairs, int cap) {
  const int b = blockIdx.z, kv = blockIdx.y, Hkv = gridDim.y;
  const int L = min(max(seq_lens[b], 0), cap);
  const int64_t t = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4;
  if (t >= L) return;
  const size_t row = (size_t)b * Hkv + kv;
  const float* lg = logits + row * pairs * (size_t)cap + t;
  f32x4 sum = {0.0f, 0.0f, 0.0f, 0.0f};
  for (int i = 0; i < pairs; ++i) {
    const f32x4 s = *reinterpret_cast<const f32x4*>(lg + (size_t)i * cap);
    const float z = lse[row * pairs + i];
#pragma unroll
    for (int e = 0; e < 4; ++e) sum[e] += exp2_(s[e] - z);
  }
  float* w = weights + row * stride + t;
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (t + e < L) w[e] += sum[e];
}

template <int D, bool BF16, bool SUMS>
hipError_t launch(const jf_kv_layout& L, const jf_kv_pool_ptrs& pool, const void* q, int32_t B,
                  int32_t sq, int32_t Hq, const int32_t* bt, int32_t max_pages, const int32_t* lens,
                  float scale, int32_t max_splits, void* ws, void* out, float* weights,
                  int64_t stride, hipStream_t stream) {
  const int Hkv = L.num_kv_heads, pairs = Hq / Hkv * sq;
  const int n_hchunks = (pairs + kCols - 1) / kCols;
  // enough blocks for one per CU when one request runs alone; the count
  // depends on neither the batch nor the lengths, so that a request's output
  // is bitwise the same in any batch
  const int split_cap = (int)std::max<int64_t>(
      1, std::min<int64_t>(max_splits, num_cus() / ((int64_t)Hkv * n_hchunks)));
  const int64_t slots = ((int64_t)split_cap * Hkv + kXcds - 1) / kXcds * kXcds;
  const Kv8Workspace at = kv8_workspace(B, sq, Hq, D, max_splits, SUMS ? max_pages * L.page_size : 0);
  uint8_t* base = static_cast<uint8_t*>(ws);
  float* lse = reinterpret_cast<float*>(base + at.lse);
  float* logits = reinterpret_cast<float*>(base + at.logits);
  int shift = 0;
  while ((1 << shift) < L.group_size) ++shift;
  const size_t lds = sizeof(float) * kWaves * std::min(kCols, pairs) * (D + 4);
  const auto kernel = kv8_decode_kernel<D, BF16, SUMS>;
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
                     max_pages, max_splits, split_cap, n_hchunks, scale * 1.44269504088896340736f);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || !SUMS) return e;
  const int cap = max_pages * L.page_size;
  hipLaunchKernelGGL(kv8_sums_kernel, dim3((uint32_t)((cap + 1023) / 1024), Hkv, B), dim3(256), 0,
                     stream, logits, lse, lens, weights, stride, pairs, cap);
  return hipGetLastError();
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
