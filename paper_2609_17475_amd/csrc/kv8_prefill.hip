// Chunk attention over the 8-bit cache (format: jfkv_kv8.h): the T rows of a
// chunk, already appended, attend causally to the prefix and to themselves,
// all read from the pages; and the sums of such rows' attention weights.
//
//   s_it = scale * q_i . k_t  (t <= prefix + i),  lse_i = log sum_t exp(s_it)
//   o_i = sum_t exp(s_it - lse_i) v_t,  w_t += sum_i exp(s_it - lse_i)
//
// Bound by the vector work beside the matrix cores, an exponential and some four
// instructions per score: at d = 128 vector instructions issue in 54 % of a SIMD's
// cycles and its matrix core is busy in 39 %, and the two hardly overlap.  The (row,
// head) pairs that read a KV head are the columns of the products, as in
// kv8_decode.hip, whose operand layouts, exponents' handling and roundings (P to fp16
// beside the values) are the same.  2,048 rows of 32/8 heads of 128 over 65,536
// positions take 2.33 ms (0.96 PFLOP/s), 256 of 24/4 heads of 256 over 196,608 1.35.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <type_traits>

#include "jfkv_internal.h"
#include "jfkv_kv8.h"

namespace jfkv {
namespace {

using namespace kv8;

#define JF_INLINE __attribute__((always_inline))

constexpr int kTile = 64;        // positions of a tile (in one page)
constexpr int kWaves = 8;
constexpr int kThreads = 64 * kWaves;
constexpr int kFar = 4;          // tiles by which lines are touched ahead of their fetch
constexpr uint32_t kZeroExp = 1;  // the exponent byte of a block of zeros
constexpr float kLog2e = 1.44269504088896340736f;

// Column sets of 16 per wave: two share every operand of K and V; at head_dim
// 256 the accumulators of one fill the registers.
template <int D>
constexpr int col_sets() {
  return D > 128 ? 1 : 2;
}
template <int D>
constexpr int block_cols() {
  return kWaves * 16 * col_sets<D>();
}

// The query row of (row, head) as B operands: dims 64 c + 16 g + 8 j ..
template <int C, bool BF16>
__device__ __forceinline__ void load_q(u32x4 (&qf)[C][2], const uint16_t* qp, int g, uint32_t flip) {
#pragma unroll
  for (int c = 0; c < C; ++c)
#pragma unroll
    for (int j = 0; j < 2; ++j)
      qf[c][j] = *reinterpret_cast<const u32x4*>(qp + 64 * c + 16 * g + 8 * j) ^ flip;
}

// One block: block_cols columns of one KV head, the tiles of one split.  A tile's
// K and V codes are fetched into registers two tiles ahead, widened once for the
// block and laid into LDS as the matrix operands that all waves read.  Several
// splits: fp32 partials (o, m, l) to ws [split][Hkv][columns][D + 4] instead of
// rows.
template <int D, bool BF16>
__global__ __launch_bounds__(kThreads) void kv8_prefill_kernel(
    const uint8_t* __restrict__ k_codes, const uint8_t* __restrict__ k_exps,
    const uint8_t* __restrict__ v_codes, const uint8_t* __restrict__ v_exps,
    const uint16_t* __restrict__ q, const int32_t* __restrict__ table, float* __restrict__ ws,
    uint16_t* __restrict__ out, float* __restrict__ lse, int Hq, int Hkv, int P, int block_shift,
    int num_pages, int T, int prefix, int n_rb, int n_split, float scale_log2, uint32_t flip) {
  constexpr int C = D / 64, NC = col_sets<D>(), COLS = block_cols<D>();
  __shared__ __align__(16) u32x4 tiles_k[2][8 * D], tiles_v[2][8 * D];
  const int tid = threadIdx.x, lane = tid & 63, n = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  // KV head fastest (one XCD's L2 sees few heads), the longest row blocks first
  const int kv = blockIdx.x % Hkv, rest = blockIdx.x / Hkv;
  const int split = rest % n_split, rb = n_rb - 1 - rest / n_split;
  const int gq = Hq / Hkv;
  const int64_t ncols = (int64_t)T * gq, col_base = (int64_t)rb * COLS;
  const int L = prefix + T;

  const int row_hi = (int)((min(col_base + COLS, ncols) - 1) / gq);
  const int64_t nt = (prefix + row_hi) / kTile + 1;
  const int j0 = (int)(nt * split / n_split), j1 = (int)(nt * (split + 1) / n_split);

  // the wave's columns
  const int64_t wcol = col_base + wave * 16 * NC;
  const bool active = wcol < ncols;
  const int w_lo = active ? (int)(wcol / gq) : 0;  // its first row
  int row[NC];
  u32x4 qf[NC][C][2];
#pragma unroll
  for (int cs = 0; cs < NC; ++cs) {
    const int64_t col = min(wcol + 16 * cs + n, ncols - 1);  // (columns past the end repeat the last)
    row[cs] = (int)(col / gq);
    load_q<C, BF16>(qf[cs], q + ((size_t)row[cs] * Hq + kv * gq + col % gq) * D, g, flip);
  }

  f32x4 acc[NC][C][4] = {};
  float m[NC], l[NC];
#pragma unroll
  for (int cs = 0; cs < NC; ++cs) m[cs] = -INFINITY, l[cs] = 0.0f;
  int e_ref = 0, e_top = -1000;

  // ---- tile transport: K's codes are fetched two tiles ahead and go to LDS one
  // tile ahead, V's one tile later each
  constexpr int kPieces = 4 * D / kThreads > 0 ? 4 * D / kThreads : 1;  // of 16 bytes per thread
  constexpr int kOf = 4 * D < kThreads ? 4 * D : kThreads;              // threads that take some
  u32x4 k_stage[kPieces], v_stage[kPieces];
  uint32_t exps = 0, exps_next = 0;  // lanes 0..3: K's exponent bytes of a tile, 4..7: V's
  // the place of a tile, stepped without divisions
  struct Place {
    int page, slot;
  };
  const int last_page = (j1 * kTile - 1) / P;
  auto step = [&](Place& at) JF_INLINE {
    at.slot += kTile;
    if (at.slot == P) at.slot = 0, ++at.page;
  };
  auto page_of = [&](const Place& at) JF_INLINE { return table[min(at.page, last_page)]; };
  // A tile without a page in the pool travels as page 0's, but counts as a tile of
  // zeros that nobody sees: page 0's codes may be NaN and its exponents are someone
  // else's.  (Its values are cleared by a mask on every tile.  Times against none at
  // all, 2,048 rows over 65,536 positions and, d = 256, 256 over 196,608: 0.96 and
  // 0.99; with a branch around the mask 1.00 and 1.02, around the products instead
  // 1.01 and 1.00.)
  auto held = [&](int pid) JF_INLINE { return (uint32_t)pid < (uint32_t)num_pages; };
  auto run_of = [&](int pid) JF_INLINE { return (size_t)((uint32_t)pid < (uint32_t)num_pages ? pid : 0) * Hkv + kv; };
  const uint32_t k_off = (tid / D * 16 + (lane & 15)) * D + tid % D / 64 * 64 + (lane >> 4) * 16;
  auto fetch_k = [&](int slot0, int pid) JF_INLINE {
    const size_t run = run_of(pid);
    const uint8_t* kp = k_codes + (run * P + slot0) * D;
    if (kOf == kThreads || tid < kOf) {
#pragma unroll
      for (int k = 0; k < kPieces; ++k)
        k_stage[k] = *reinterpret_cast<const u32x4*>(kp + k_off + k * (kThreads / D) * 16 * D);
    }
    const uint8_t* ep = (lane & 4) ? v_exps : k_exps;
    exps_next = ep[run * (P >> block_shift) + ((slot0 + 16 * (lane & 3)) >> block_shift)];
  };
  auto fetch_v = [&](int slot0, int pid) JF_INLINE {
    const uint8_t* vp = v_codes + (run_of(pid) * P + slot0) * D;
    if (kOf == kThreads || tid < kOf) {
#pragma unroll
      for (int k = 0; k < kPieces; ++k)
        v_stage[k] = *reinterpret_cast<const u32x4*>(vp + (tid + k * kThreads) * 16);
    }
  };
  auto deposit_k = [&](int j) JF_INLINE {
    if (kOf < kThreads && tid >= kOf) return;
#pragma unroll
    for (int k = 0; k < kPieces; ++k) {
      const int i = tid + k * kThreads;
      // [16 positions][64 dims][half][lane]
      u32x4* to = tiles_k[j & 1] + i / 64 * 128 + i % 64;
      to[0] = widen8<BF16>(k_stage[k].x, k_stage[k].y), to[64] = widen8<BF16>(k_stage[k].z, k_stage[k].w);
    }
  };
  auto deposit_v = [&](int j, uint32_t keep) JF_INLINE {  // keep: all ones, or 0 without a page
    if (kOf < kThreads && tid >= kOf) return;
#pragma unroll
    for (int k = 0; k < kPieces; ++k) {
      const int i = tid + k * kThreads;
      v_stage[k] &= keep;
      if ((j + 1) * kTile > L) {  // slots not written yet: zeros (their codes may be NaN)
        const int left = min(max(L - (j * kTile + i / D * 16 + i % 64 / 16 * 4), 0), 4);
        v_stage[k] &= left ? 0xffffffffu >> (8 * (4 - left)) : 0u;
      }
      // [32 positions][64 dims][dim % 4][lane][16 of the 32]
      u32x2* to = reinterpret_cast<u32x2*>(tiles_v[j & 1] + (i / D / 2 * C + i % D / 64) * 256 + i % 64) + i / D % 2;
#pragma unroll
      for (int dt = 0; dt < 4; ++dt) {
        uint32_t lo, hi;
        widen<false>(v_stage[k][dt], lo, hi);
        to[dt * 128] = u32x2{lo, hi};
      }
    }
  };

  auto rescale = [&](float f) JF_INLINE {
#pragma unroll
    for (int cs = 0; cs < NC; ++cs)
#pragma unroll
      for (int c = 0; c < C; ++c)
#pragma unroll
        for (int dt = 0; dt < 4; ++dt) acc[cs][c][dt] *= f;
  };

  // ---- a tile's three steps: scores (matrix cores), softmax (vector), values
  // (matrix cores)
  f32x4 s[4][NC];      // scores, times f[t] in log2 units
  float f[4];
  int ev[4];           // the values' exponents
  uint32_t pf[2][NC][4];  // P as B operands
  int split_e[4];      // where apart: the references of the tile's parts
  bool apart = false;

  // A run of operands that lie one after the other in LDS, each read kAhead
  // before its products.  (The barriers keep the compiler from reading all of
  // them at once, which spills.)
  constexpr int kAhead = 4;
  auto stream = [&](const u32x4* from, auto first, auto count, auto&& use) JF_INLINE {
    constexpr int n0 = decltype(first)::value, nn = decltype(count)::value;
    u32x4 ring[kAhead];
#pragma unroll
    for (int p = 0; p < kAhead; ++p) ring[p] = from[(n0 + p) * 64 + lane];
#pragma unroll
    for (int p = 0; p < nn; ++p) {
      const u32x4 a = ring[p % kAhead];
      if (p + kAhead < nn) ring[p % kAhead] = from[(n0 + p + kAhead) * 64 + lane];
      use(n0 + p, a);
      __builtin_amdgcn_sched_barrier(0);
    }
  };

  auto scores = [&](int j) JF_INLINE {
#pragma unroll
    for (int t = 0; t < 4; ++t) {
#pragma unroll
      for (int cs = 0; cs < NC; ++cs) s[t][cs] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
      // (not 0, so that a hidden score times it stays -inf)
      f[t] = fmaxf(scale_log2 * power2(__builtin_amdgcn_readlane((int)exps, t) - 127), 1e-37f);
      ev[t] = __builtin_amdgcn_readlane((int)exps, 4 + t) - 127;
    }
    stream(tiles_k[j & 1], std::integral_constant<int, 0>{}, std::integral_constant<int, 8 * C>{},
           [&](int p, u32x4 a) JF_INLINE {
             const int t = p / (2 * C), c = p / 2 % C, half = p % 2;
#pragma unroll
             for (int cs = 0; cs < NC; ++cs) s[t][cs] = mma<BF16>(a, qf[cs][c][half], s[t][cs]);
           });
  };

  auto softmax = [&](int j, bool on) JF_INLINE {
    const int pos0 = j * kTile;
    if (!on || pos0 + kTile - 1 > prefix + w_lo) {
#pragma unroll
      for (int t = 0; t < 4; ++t) {
#pragma unroll
        for (int cs = 0; cs < NC; ++cs)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (!on || pos0 + 16 * t + 4 * g + i > prefix + row[cs]) s[t][cs][i] = -INFINITY;
        if (pos0 + 16 * t >= L) f[t] = 1.0f, ev[t] = ev[0];  // (exponents not written yet)
      }
    }
    // maxima
    float top[NC];
    bool raise = false;
#pragma unroll
    for (int cs = 0; cs < NC; ++cs) {
      top[cs] = -INFINITY;
#pragma unroll
      for (int t = 0; t < 4; ++t)
        top[cs] = larger(top[cs], f[t] * larger(larger(larger(s[t][cs][0], s[t][cs][1]),
                                                       s[t][cs][2]), s[t][cs][3]));
      raise |= top[cs] > m[cs] + kMargin;
    }
    if (__any(raise)) {
#pragma unroll
      for (int cs = 0; cs < NC; ++cs) {
        const float mn = fmaxf(m[cs], col_max(top[cs]));
        const float by = m[cs] == -INFINITY ? 0.0f : exp2_(m[cs] - mn);
        l[cs] *= by;
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
          for (int dt = 0; dt < 4; ++dt) acc[cs][c][dt] *= by;
        m[cs] = mn;
      }
    }
    float mu[NC];
#pragma unroll
    for (int cs = 0; cs < NC; ++cs) mu[cs] = m[cs] == -INFINITY ? 0.0f : m[cs];
    int lo = ev[0], hi = ev[0];
#pragma unroll
    for (int t = 1; t < 4; ++t) lo = min(lo, ev[t]), hi = max(hi, ev[t]);
    e_top = max(e_top, hi);
    apart = hi - lo > kRefMax || lo < e_top - kRefFloor;
    if (!apart) {
      // one reference for the tile's values
      if (lo < e_ref || hi > e_ref + kRefMax) {
        const int e = max(hi - kRefMax, lo - 4);
        rescale(reference_step(e_ref, e));
        e_ref = e;
      }
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int cs = 0; cs < NC; ++cs) {
          const float by = (float)(ev[t] - e_ref) - mu[cs];
          float p[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) p[i] = exp2_(fmaf(s[t][cs][i], f[t], by));
          l[cs] = fmaf((p[0] + p[1]) + (p[2] + p[3]), power2(e_ref - ev[t]), l[cs]);
          pf[t / 2][cs][t % 2 * 2] = narrow2<false>(p[0], p[1]);
          pf[t / 2][cs][t % 2 * 2 + 1] = narrow2<false>(p[2], p[3]);
        }
    } else {
      // too far apart for that (or far below the largest values, where P may
      // vanish and l must not): a reference for each 16 positions
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        split_e[t] = max(ev[t] - 4, e_top - kRefFloor);
#pragma unroll
        for (int cs = 0; cs < NC; ++cs) {
          const float by = (float)(ev[t] - split_e[t]) - mu[cs];
          float p[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float x = s[t][cs][i] * f[t];
            p[i] = exp2_(x + by);
            l[cs] += exp2_(x - mu[cs]);
          }
          pf[t / 2][cs][t % 2 * 2] = narrow2<false>(p[0], p[1]);
          pf[t / 2][cs][t % 2 * 2 + 1] = narrow2<false>(p[2], p[3]);
        }
      }
    }
  };

  auto values = [&](int j) JF_INLINE {
    auto products = [&](auto t2, const u32x4 (&b)[NC]) {
      stream(tiles_v[j & 1], std::integral_constant<int, decltype(t2)::value * 4 * C>{},
             std::integral_constant<int, 4 * C>{}, [&](int p, u32x4 a) JF_INLINE {
               const int c = p / 4 % C, dt = p % 4;
#pragma unroll
               for (int cs = 0; cs < NC; ++cs) acc[cs][c][dt] = mma<false>(a, b[cs], acc[cs][c][dt]);
             });
    };
    constexpr std::integral_constant<int, 0> t0{};
    constexpr std::integral_constant<int, 1> t1{};
    if (!apart) {
#pragma unroll
      for (int t2 = 0; t2 < 2; ++t2) {
        u32x4 b[NC];
#pragma unroll
        for (int cs = 0; cs < NC; ++cs) b[cs] = u32x4{pf[t2][cs][0], pf[t2][cs][1], pf[t2][cs][2], pf[t2][cs][3]};
        if (t2 == 0) products(t0, b); else products(t1, b);
      }
    } else {
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        rescale(reference_step(e_ref, split_e[t]));
        e_ref = split_e[t];
        u32x4 b[NC];
#pragma unroll
        for (int cs = 0; cs < NC; ++cs)
          b[cs] = t % 2 ? u32x4{0u, 0u, pf[t / 2][cs][2], pf[t / 2][cs][3]}
                        : u32x4{pf[t / 2][cs][0], pf[t / 2][cs][1], 0u, 0u};
        if (t < 2) products(t0, b); else products(t1, b);
      }
    }
  };

  // ---- Turn j forms the scores of tile j and the value products of tile j - 1.
  // Waves w and w + 4 share a SIMD: the first do their matrix products at once and
  // the vector work (the softmax, the next tiles' way into LDS) after them, the
  // second the other way round, so that one's matrix products meet the other's
  // vector work (d = 256: 256 rows over 196,608 positions 1,790 -> 1,430 us; at d =
  // 64, where the vector work is the most, all do the same).  (Two loops, as one loop
  // with both orders spills; every wave passes j1 - j0 + 1 barriers in either.)
  auto walk = [&](auto is_late) JF_INLINE {
    constexpr bool late = decltype(is_late)::value;
    Place at = {j0 * kTile / P, j0 * kTile % P};
    int pid[4], slot[4];  // of tiles j - 1, j, j + 1, j + 2
    pid[0] = -1, slot[0] = 0;
#pragma unroll
    for (int i = 1; i < 4; ++i) {
      pid[i] = page_of(at), slot[i] = at.slot;
      step(at);
    }
    fetch_k(slot[1], pid[1]);
    exps = held(pid[1]) ? exps_next : kZeroExp;
    deposit_k(j0);
    fetch_v(slot[1], pid[1]);
    fetch_k(slot[2], pid[2]);
    // kFar tiles further ahead each line is touched once, so that the fetches find
    // it in the L2 (2,048 rows over 65,536 positions that the last-level cache does
    // not hold: 2,815 -> 2,540 us)
    Place far = at;
#pragma unroll
    for (int i = 0; i < kFar; ++i) step(far);
    int pid_far = page_of(far), slot_far = far.slot;
    uint32_t touched = 0;
    for (int j = j0; j <= j1; ++j) {
      __syncthreads();  // K of tile j and V of tile j - 1 are in LDS
      const int pid_n = page_of(at);
      if (tid < D) {
        asm volatile("" ::"v"(touched));
        const uint8_t* from = (tid < D / 2 ? k_codes : v_codes) + (run_of(pid_far) * P + slot_far) * D;
        touched = *reinterpret_cast<const uint32_t*>(from + tid % (D / 2) * 128);
      }
      step(far);
      pid_far = page_of(far), slot_far = far.slot;
      uint32_t exps_1 = exps_next;
      auto transport = [&]() JF_INLINE {
        if (j < j1) {
          deposit_v(j, held(pid[1]) ? 0xffffffffu : 0u);
          fetch_v(slot[2], pid[2]);
        }
        if (j + 1 < j1) {
          deposit_k(j + 1);
          fetch_k(slot[3], pid[3]);
        }
      };
      if constexpr (late) {
        if (active && j > j0) softmax(j - 1, (uint32_t)pid[0] < (uint32_t)num_pages);
        transport();
      }
      __builtin_amdgcn_s_setprio(1);
      if (active) {
        if (j > j0) values(j - 1);
        if (j < j1) scores(j);
      }
      __builtin_amdgcn_s_setprio(0);
      if constexpr (!late) {
        if (active && j < j1) softmax(j, (uint32_t)pid[1] < (uint32_t)num_pages);
        transport();
      }
      exps = held(pid[2]) ? exps_1 : kZeroExp;
#pragma unroll
      for (int i = 0; i < 3; ++i) pid[i] = pid[i + 1], slot[i] = slot[i + 1];
      pid[3] = pid_n, slot[3] = at.slot;
      step(at);
    }
  };
  if (j0 < j1) {
    if (D > 64 && wave >= kWaves / 2)
      walk(std::true_type{});
    else
      walk(std::false_type{});
  }

  // ---- rows out, or partials
  if (!active) return;
  const float unit = __builtin_ldexpf(1.0f, e_ref);
#pragma unroll
  for (int cs = 0; cs < NC; ++cs) {
    const float den = col_sum(l[cs]);
    const int64_t col = wcol + 16 * cs + n;
    if (col >= ncols) continue;
    if (n_split == 1) {
      const float r = den > 0.0f ? unit / den : 0.0f;
      const size_t at = (size_t)row[cs] * Hq + kv * gq + col % gq;
      uint16_t* op = out + at * D + 16 * g;
#pragma unroll
      for (int c = 0; c < C; ++c)
#pragma unroll
        for (int i = 0; i < 4; i += 2) {
          const f32x4(&a)[4] = acc[cs][c];
          *reinterpret_cast<uint4*>(op + 64 * c + 4 * i) =
              make_uint4(narrow2<BF16>(a[0][i] * r, a[1][i] * r),
                         narrow2<BF16>(a[2][i] * r, a[3][i] * r),
                         narrow2<BF16>(a[0][i + 1] * r, a[1][i + 1] * r),
                         narrow2<BF16>(a[2][i + 1] * r, a[3][i + 1] * r));
        }
      if (lse && g == 0)
        lse[at] = den > 0.0f ? (m[cs] + __log2f(den)) * (1.0f / kLog2e) : -INFINITY;
    } else {
      float* rec = ws + (((size_t)split * Hkv + kv) * ncols + col) * (D + 4);
#pragma unroll
      for (int c = 0; c < C; ++c)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          *reinterpret_cast<f32x4*>(rec + 64 * c + 16 * g + 4 * i) =
              f32x4{acc[cs][c][0][i], acc[cs][c][1][i], acc[cs][c][2][i], acc[cs][c][3][i]} * unit;
      if (g == 0) rec[D] = m[cs], rec[D + 1] = den;
    }
  }
}

// Joins the splits' partials: a thread takes four dims of one column.
template <int D, bool BF16>
__global__ __launch_bounds__(256) void kv8_prefill_combine_kernel(
    const float* __restrict__ ws, uint16_t* __restrict__ out, float* __restrict__ lse, int Hq,
    int Hkv, int64_t ncols, int n_split) {
  const int gq = Hq / Hkv;
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int64_t at = i / (D / 4);  // (KV head, column)
  const int d4 = (int)(i % (D / 4));
  if (at >= ncols * Hkv) return;
  float M = -INFINITY, den = 0.0f;
  f32x4 num = {0.0f, 0.0f, 0.0f, 0.0f};
  for (int s = 0; s < n_split; ++s) {
    const float* rec = ws + ((size_t)s * Hkv * ncols + at) * (D + 4);
    const float ms = rec[D], mx = fmaxf(M, ms);
    const f32x4 o = *reinterpret_cast<const f32x4*>(rec + 4 * d4);
    const float a = M == -INFINITY ? 0.0f : exp2_(M - mx), b = ms == -INFINITY ? 0.0f : exp2_(ms - mx);
    num = num * a + o * b;
    den = den * a + rec[D + 1] * b;
    M = mx;
  }
  const float r = den > 0.0f ? 1.0f / den : 0.0f;
  const int64_t kv = at / ncols, col = at % ncols;
  const size_t dst = (size_t)(col / gq) * Hq + kv * gq + col % gq;
  *reinterpret_cast<uint2*>(out + dst * D + 4 * d4) =
      make_uint2(narrow2<BF16>(num.x * r, num.y * r), narrow2<BF16>(num.z * r, num.w * r));
  if (lse && d4 == 0) lse[dst] = den > 0.0f ? (M + __log2f(den)) * (1.0f / kLog2e) : -INFINITY;
}

// ---- attention weights of a chunk's rows, added up per position
//
// A wave owns 16 NS positions, whose K it holds as matrix operands in
// registers, and walks over all columns that see them; the columns' queries
// (B operands) and (lse, row) pass through LDS, shared by the block's four
// waves.  No two waves add to the same position, so the sums' order is fixed.
// Weights are never rounded below fp32.  Bound by the matrix cores (2 d flops per
// score), and at d <= 128 as much by the vector work (an exponential, a fused
// product and a sum per score); K is read once, Q once per 64 NS positions (from
// the L2 of the head's XCD).
constexpr int kWWaves = 4;
constexpr int kWThreads = 64 * kWWaves;

// a + b columns, as (row, head) with head < gq
struct Column {
  int row, head;
  __device__ __forceinline__ void advance(int rows, int heads, int gq) {
    row += rows, head += heads;
    if (head >= gq) head -= gq, ++row;
  }
};

template <int D, bool BF16, int NS>
__global__ __launch_bounds__(kWThreads, NS > 2 ? 2 : 3) void kv8_weights_kernel(
    const uint8_t* __restrict__ k_codes, const uint8_t* __restrict__ k_exps,
    const uint16_t* __restrict__ q, const float* __restrict__ lse,
    const int32_t* __restrict__ table, float* __restrict__ weights, int64_t stride, int Hq, int Hkv,
    int P, int block_shift, int num_pages, int T, int prefix, float scale_log2) {
  constexpr int C = D / 64, kCols = D > 128 ? 32 : 64;  // columns in LDS at a time
  constexpr int kItems = kCols * D * 2 / 16 / kWThreads;
  constexpr int kEvery = C > 2 ? C / 2 : 1;              // items of a thread in one group of 16 columns
  constexpr int kStep = C > 2 ? 16 : 16 * 2 / C;         // columns from one such run to the next
  __shared__ __align__(16) u32x4 qs[2][kCols * D / 8];   // [16 columns][c][half][lane]
  __shared__ float s_lse[2][kCols];
  __shared__ int s_row[2][kCols];
  const int tid = threadIdx.x, lane = tid & 63, n = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int kv = blockIdx.x % Hkv, gq = Hq / Hkv;
  const int ncols = T * gq;
  const int L = prefix + T;
  const int64_t base = (int64_t)(blockIdx.x / Hkv) * (kWWaves * 16 * NS);
  const int64_t key0_64 = base + wave * 16 * NS;
  const bool mine = key0_64 < L;
  const int key0 = mine ? (int)key0_64 : 0;

  // the wave's keys as A operands, and their factors
  const int pid = table[key0 / P];
  const bool on = mine && (uint32_t)pid < (uint32_t)num_pages;
  const size_t run = (size_t)(on ? pid : 0) * Hkv + kv;
  const int slot0 = key0 % P;
  u32x4 kf[NS][C][2];
  float f[NS];
#pragma unroll
  for (int t = 0; t < NS; ++t) {
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const u32x4 kc = *reinterpret_cast<const u32x4*>(k_codes + (run * P + slot0 + 16 * t + n) * D +
                                                       64 * c + 16 * g);
      kf[t][c][0] = widen8<BF16>(kc.x, kc.y), kf[t][c][1] = widen8<BF16>(kc.z, kc.w);
    }
    f[t] = scale_log2 * power2((int)k_exps[run * (P >> block_shift) + ((slot0 + 16 * t) >> block_shift)] - 127);
  }
  float w[NS][4] = {};

  // columns from the first row that sees the block's first key; (row, head) of the
  // columns that this thread brings to LDS are stepped without divisions
  const int col0 = (int)(max((int64_t)0, base - prefix) * gq / kCols * kCols);
  const int step_r = kStep / gq, step_h = kStep % gq, lse_r = kCols / gq, lse_h = kCols % gq;
  Column qc, lc;
  {
    const int c = col0 + 16 * (wave / (2 * C)) + n, d = col0 + tid % kCols;
    qc = {c / gq, c % gq}, lc = {d / gq, d % gq};
  }
  // what a thread brings to LDS for one turn; two turns are on their way
  struct Stage {
    u32x4 x[kItems];
    float lse;
    int row;
  };
  const uint16_t* const qh = q + (size_t)kv * gq * D + 16 * g;
  auto fetch = [&](Stage& st) JF_INLINE {
#pragma unroll
    for (int k = 0; k < kItems; ++k) {
      const int cj = (wave + kWWaves * k) % (2 * C);
      st.x[k] = *reinterpret_cast<const u32x4*>(
          qh + ((size_t)min(qc.row, T - 1) * Hq + qc.head) * D + 64 * (cj >> 1) + 8 * (cj & 1));
      if ((k + 1) % kEvery == 0) qc.advance(step_r, step_h, gq);
    }
    st.row = lc.row;
    if (tid < kCols) {
      st.lse = lse[(size_t)min(lc.row, T - 1) * Hq + kv * gq + lc.head];
      lc.advance(lse_r, lse_h, gq);
    }
  };
  auto turn = [&](Stage& st, int buf) JF_INLINE {
#pragma unroll
      for (int k = 0; k < kItems; ++k) qs[buf][tid + k * kWThreads] = st.x[k];
      if (tid < kCols) {
        // a row that sees nothing, and columns past the end, weigh nothing
        s_lse[buf][tid] = st.row < T && st.lse != -INFINITY ? st.lse * kLog2e : INFINITY;
        s_row[buf][tid] = min(st.row, T - 1);
      }
      __syncthreads();
      fetch(st);
      if (!on) return;
      // whether all columns of the stage see all of the wave's keys (rows ascend)
      const bool whole = key0 + 16 * NS - 1 <= prefix + __builtin_amdgcn_readfirstlane(s_row[buf][0]);
#pragma unroll
      for (int grp = 0; grp < kCols / 16; grp += 2) {
        f32x4 s[2][NS];
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int t = 0; t < NS; ++t) s[u][t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
          for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int u = 0; u < 2; ++u) {
              const u32x4 b = qs[buf][(((grp + u) * C + c) * 2 + j) * 64 + lane];
#pragma unroll
              for (int t = 0; t < NS; ++t) s[u][t] = mma<BF16>(kf[t][c][j], b, s[u][t]);
            }
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const float z = s_lse[buf][16 * (grp + u) + n];
          if (!whole) {
            const int see = prefix + s_row[buf][16 * (grp + u) + n];  // the last position the column sees
#pragma unroll
            for (int t = 0; t < NS; ++t)
#pragma unroll
              for (int i = 0; i < 4; ++i)
                w[t][i] += key0 + 16 * t + 4 * g + i > see ? 0.0f : exp2_(fmaf(s[u][t][i], f[t], -z));
          } else {
#pragma unroll
            for (int t = 0; t < NS; ++t)
#pragma unroll
              for (int i = 0; i < 4; ++i) w[t][i] += exp2_(fmaf(s[u][t][i], f[t], -z));
          }
        }
      }
  };
  if (col0 < ncols) {
    Stage s0, s1;
    fetch(s0);
    fetch(s1);
    for (int at = col0; at < ncols; at += 2 * kCols) {
      turn(s0, 0);
      if (at + kCols < ncols) turn(s1, 1);
    }
  }
  if (!on) return;
  // Sums over the 16 lanes that share the positions: halved turn by turn, until
  // lane n holds the sum of position 16 (n / 4) + 4 g + n % 4.  (Written out in both
  // kernels: as a function of w it takes registers, and at d = 256 spills, more.)
  float v[4 * NS];
#pragma unroll
  for (int i = 0; i < 4 * NS; ++i) v[i] = w[i / 4][i % 4];
#pragma unroll
  for (int o = 2 * NS; o; o >>= 1)
#pragma unroll
    for (int k = 0; k < o; ++k) {
      const bool up = (n & o) != 0;
      v[k] = (up ? v[k + o] : v[k]) + __shfl_xor(up ? v[k] : v[k + o], o);
    }
  if (NS == 2) v[0] += __shfl_xor(v[0], 8);
  const int pos = key0 + 16 * (n / 4) + 4 * g + n % 4;
  if (n < 4 * NS && pos < L) weights[(size_t)kv * stride + pos] += v[0];
}

// The same where all columns' queries fit into LDS (an observation window): they
// are brought there once, and a block per CU walks over the positions of its KV
// head, each wave over its own 64 at a time without a barrier, the next ones' K on
// the way meanwhile.
constexpr int kWinWaves = 8;
constexpr int kWinThreads = 64 * kWinWaves;
constexpr int kWinNS = 4;
template <int D>
constexpr size_t window_bytes(int64_t ncols) {  // (whole pairs of groups of 16)
  return (size_t)((ncols + 31) / 32 * 32) * (2 * D + 8);
}
constexpr size_t kWindowMax = 147456;

template <int D, bool BF16>
__global__ __launch_bounds__(kWinThreads) void kv8_window_weights_kernel(
    const uint8_t* __restrict__ k_codes, const uint8_t* __restrict__ k_exps,
    const uint16_t* __restrict__ q, const float* __restrict__ lse,
    const int32_t* __restrict__ table, float* __restrict__ weights, int64_t stride, int Hq, int Hkv,
    int P, int block_shift, int num_pages, int T, int prefix, float scale_log2, uint32_t flip) {
  constexpr int C = D / 64, NS = kWinNS;
  constexpr bool kAheadK = D <= 128;  // (the registers do not hold two sets of d = 256)
  extern __shared__ __align__(16) u32x4 qs[];  // [16 columns][c][half][lane], lse, row
  const int tid = threadIdx.x, lane = tid & 63, n = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int kv = blockIdx.x % Hkv, gq = Hq / Hkv, ncols = T * gq, pairs = (ncols + 31) / 32;
  float* const s_lse = reinterpret_cast<float*>(qs + pairs * 32 * (D / 8));
  int* const s_row = reinterpret_cast<int*>(s_lse + pairs * 32);
  const int L = prefix + T, units = (L + 16 * NS - 1) / (16 * NS);
  const int stepu = gridDim.x / Hkv * kWinWaves;
  const int last = units - 1;

  u32x4 kc[NS][C];
  uint32_t ke[NS];
  auto page_of = [&](int u) JF_INLINE { return table[min(u, last) * (16 * NS) / P]; };
  auto fetch = [&](int u, int pid) JF_INLINE {
    const size_t run = (size_t)((uint32_t)pid < (uint32_t)num_pages ? pid : 0) * Hkv + kv;
    const int slot0 = min(u, last) * (16 * NS) % P;
#pragma unroll
    for (int t = 0; t < NS; ++t) {
#pragma unroll
      for (int c = 0; c < C; ++c)
        kc[t][c] = *reinterpret_cast<const u32x4*>(k_codes + (run * P + slot0 + 16 * t + n) * D +
                                                   64 * c + 16 * g);
      ke[t] = k_exps[run * (P >> block_shift) + ((slot0 + 16 * t) >> block_shift)];
    }
  };
  int u = blockIdx.x / Hkv * kWinWaves + wave;
  int pid = page_of(u), pid_next = page_of(u + stepu);
  if (kAheadK) fetch(u, pid);

  // ---- all columns to LDS; those past the end weigh nothing
  const int count = pairs * 32 * (D / 8);
  for (int i0 = tid; i0 < count; i0 += 8 * kWinThreads) {
    u32x4 x[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const int i = min(i0 + k * kWinThreads, count - 1), col = min(i / (128 * C) * 16 + i % 16, ncols - 1);
      x[k] = *reinterpret_cast<const u32x4*>(
          q + ((size_t)(col / gq) * Hq + kv * gq + col % gq) * D + i / 128 % C * 64 +
          i % 64 / 16 * 16 + i / 64 % 2 * 8);
    }
#pragma unroll
    for (int k = 0; k < 8; ++k)
      if (i0 + k * kWinThreads < count) qs[i0 + k * kWinThreads] = x[k] ^ flip;
  }
  for (int col = tid; col < pairs * 32; col += kWinThreads) {
    const int row = min(col, ncols - 1) / gq;
    const float z = lse[(size_t)row * Hq + kv * gq + min(col, ncols - 1) % gq];
    s_lse[col] = col < ncols && z != -INFINITY ? z * kLog2e : INFINITY;
    s_row[col] = row;
  }
  __syncthreads();

  // ---- 32 columns against the wave's positions: the products of one pair of
  // groups, and between them the exponentials of the pair before
  struct Scores {
    f32x4 s[2][NS];
    float z[2];
  };
  u32x4 kf[NS][C][2];
  float f[NS], w[NS][4];
  auto one = [&](const Scores& a, int i) JF_INLINE {  // score i of 32
    const int h = i / (4 * NS), t = i / 4 % NS, e = i % 4;
    w[t][e] += exp2_(fmaf(a.s[h][t][e], f[t], -a.z[h]));
  };
  auto weigh = [&](const Scores& a) JF_INLINE {
#pragma unroll
    for (int i = 0; i < 8 * NS; ++i) one(a, i);
  };
  auto step = [&](int p, Scores& now, const Scores& before, auto both) JF_INLINE {
    constexpr int kOps = 4 * C, kAhead = 4, kPer = 8 * NS / kOps;
    const u32x4* const from = qs + p * 32 * (D / 8) + lane;
    u32x4 ring[kAhead];
#pragma unroll
    for (int o = 0; o < kAhead; ++o) ring[o] = from[o * 64];
    now.z[0] = s_lse[32 * p + n], now.z[1] = s_lse[32 * p + 16 + n];
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int t = 0; t < NS; ++t) now.s[h][t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int o = 0; o < kOps; ++o) {  // (in the order of LDS: [h][c][half])
      const u32x4 x = ring[o % kAhead];
      if (o + kAhead < kOps) ring[o % kAhead] = from[(o + kAhead) * 64];
      const int h = o / (2 * C), c = o / 2 % C, j = o % 2;
#pragma unroll
      for (int t = 0; t < NS; ++t) now.s[h][t] = mma<BF16>(kf[t][c][j], x, now.s[h][t]);
      if constexpr (decltype(both)::value) {
#pragma unroll
        for (int i = 0; i < kPer; ++i) one(before, o * kPer + i);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  Scores scored, spare;

  for (; u < units; u += stepu) {
    if (!kAheadK) fetch(u, pid);
    const int key0 = u * (16 * NS), pos = key0 + 16 * (n / 4) + 4 * g + n % 4;
    const float old = weights[(size_t)kv * stride + min(pos, L - 1)];
    const bool on = (uint32_t)pid < (uint32_t)num_pages;
#pragma unroll
    for (int t = 0; t < NS; ++t) {
#pragma unroll
      for (int c = 0; c < C; ++c) {
        kf[t][c][0] = widen8<BF16>(kc[t][c].x, kc[t][c].y);
        kf[t][c][1] = widen8<BF16>(kc[t][c].z, kc[t][c].w);
      }
      // (not 0, so that a hidden score times it stays -inf)
      f[t] = fmaxf(scale_log2 * power2((int)ke[t] - 127), 1e-37f);
#pragma unroll
      for (int i = 0; i < 4; ++i) w[t][i] = 0.0f;
    }
    pid = pid_next;
    if (kAheadK) fetch(u + stepu, pid);
    pid_next = page_of(u + 2 * stepu);
    if (!on) continue;
    if (key0 + 16 * NS - 1 > prefix) {  // (some rows do not see all of these positions)
      for (int p = 0; p < pairs; ++p) {
        step(p, scored, spare, std::false_type{});
        const int see0 = prefix + s_row[32 * p + n], see1 = prefix + s_row[32 * p + 16 + n];
#pragma unroll
        for (int t = 0; t < NS; ++t)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int pos = key0 + 16 * t + 4 * g + i;
            if (pos > see0) scored.s[0][t][i] = -INFINITY;
            if (pos > see1) scored.s[1][t][i] = -INFINITY;
          }
        weigh(scored);
      }
    } else {
      step(0, scored, spare, std::false_type{});
      int p = 1;
      for (; p + 1 < pairs; p += 2) {
        step(p, spare, scored, std::true_type{});
        step(p + 1, scored, spare, std::true_type{});
      }
      if (p < pairs) {
        step(p, spare, scored, std::true_type{});
        weigh(spare);
      } else {
        weigh(scored);
      }
    }
    float v[4 * NS];  // (as above: lane n gets the sum of its position)
#pragma unroll
    for (int i = 0; i < 4 * NS; ++i) v[i] = w[i / 4][i % 4];
#pragma unroll
    for (int o = 2 * NS; o; o >>= 1)
#pragma unroll
      for (int k = 0; k < o; ++k) {
        const bool up = (n & o) != 0;
        v[k] = (up ? v[k + o] : v[k]) + __shfl_xor(up ? v[k] : v[k + o], o);
      }
    if (pos < L) weights[(size_t)kv * stride + pos] = old + v[0];
  }
}

template <int D, bool BF16>
hipError_t launch_prefill_t(const jf_kv_layout& L, const jf_kv_pool_ptrs& pool, const void* q,
                            int32_t T, int32_t Hq, const int32_t* table, int32_t prefix,
                            float scale, int n_split, float* ws, void* out, float* lse, int shift,
                            hipStream_t stream) {
  const int Hkv = L.num_kv_heads;
  const int64_t ncols = (int64_t)T * (Hq / Hkv);
  const int n_rb = (int)((ncols + block_cols<D>() - 1) / block_cols<D>());
  // a negative scale negates the queries, so that the scores' factors are positive
  hipLaunchKernelGGL((kv8_prefill_kernel<D, BF16>), dim3((uint32_t)(Hkv * (int64_t)n_rb * n_split)),
                     dim3(kThreads), 0, stream, static_cast<const uint8_t*>(pool.k_codes),
                     static_cast<const uint8_t*>(pool.k_meta),
                     static_cast<const uint8_t*>(pool.v_codes),
                     static_cast<const uint8_t*>(pool.v_meta), static_cast<const uint16_t*>(q),
                     table, ws, static_cast<uint16_t*>(out), lse, Hq, Hkv, L.page_size, shift,
                     L.num_pages, T, prefix, n_rb, n_split, std::fabs(scale) * kLog2e,
                     scale < 0.0f ? 0x80008000u : 0u);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || n_split == 1) return e;
  const int64_t threads = ncols * Hkv * (D / 4);
  hipLaunchKernelGGL((kv8_prefill_combine_kernel<D, BF16>), dim3((uint32_t)((threads + 255) / 256)),
                     dim3(256), 0, stream, ws, static_cast<uint16_t*>(out), lse, Hq, Hkv, ncols,
                     n_split);
  return hipGetLastError();
}

int shift_of(int block) {
  int s = 0;
  while ((1 << s) < block) ++s;
  return s;
}

}  // namespace

// Splits of a chunk's tiles: the count with the least estimated time.  A turn
// of the chip takes the tiles of its longest block and a start and end worth
// about four; the partials are written and read once, at about 4 TB/s, and
// joined by a second launch, at a tile's 1.7 us.  (That is what a tile takes at d =
// 64; it takes 2.1-2.2 at 128 and 256.  With these a tenth of all shapes are cut
// differently, few of them for more than a microsecond: at d = 128 some short chunks
// without a prefix gain, 304 rows of 8/8 heads 20.2 -> 17.9 us, others lose, 115 of
// 16/4 over 1,255 23.6 -> 24.4.)
int kv8_prefill_splits(const jf_kv_layout& L, int32_t T, int32_t Hq, int32_t prefix) {
  const int cols = L.head_dim == 256 ? block_cols<256>() : L.head_dim == 128 ? block_cols<128>() : block_cols<64>();
  const int64_t ncols = (int64_t)T * (Hq / L.num_kv_heads);
  const int64_t blocks = (ncols + cols - 1) / cols * L.num_kv_heads, cus = num_cus();
  const int64_t tiles = ((int64_t)prefix + T - 1) / kTile + 1;
  int best = 1;
  double least = 0.0;
  for (int s = 1; s <= 64 && s <= tiles; ++s) {
    const double turns = (double)((blocks * s + cus - 1) / cus);
    double cost = turns * ((double)((tiles + s - 1) / s) + 4.0);
    if (s > 1) cost += 2.0 + (double)s * ncols * L.num_kv_heads * (L.head_dim + 4) * 8.0 / 4e12 / 1.7e-6;
    if (s == 1 || cost < 0.98 * least) least = cost, best = s;
  }
  return best;
}

size_t kv8_prefill_bytes(const jf_kv_layout& L, int32_t T, int32_t Hq, int splits) {
  return splits <= 1 ? 0 : (size_t)splits * T * Hq * (L.head_dim + 4) * sizeof(float);
}

hipError_t launch_kv8_prefill(const jf_kv_layout& L, const jf_kv_pool_ptrs& pool, bool bf16,
                              const void* q, int32_t T, int32_t Hq, const int32_t* block_table,
                              int32_t prefix_len, float softmax_scale, int splits, void* ws,
                              void* out, float* lse, hipStream_t stream) {
  auto go = [&](auto fn) {
    return fn(L, pool, q, T, Hq, block_table, prefix_len, softmax_scale, splits,
              static_cast<float*>(ws), out, lse, shift_of(L.group_size), stream);
  };
  if (L.head_dim == 64) return bf16 ? go(launch_prefill_t<64, true>) : go(launch_prefill_t<64, false>);
  if (L.head_dim == 128) return bf16 ? go(launch_prefill_t<128, true>) : go(launch_prefill_t<128, false>);
  return bf16 ? go(launch_prefill_t<256, true>) : go(launch_prefill_t<256, false>);
}

namespace {
// Windows whose queries fit into LDS, where (nearly, 31 of 32) every wave has a unit
// of positions to walk over; at d = 256, where K is not fetched ahead, two.  The
// window / the kernel above, 64 rows of 32/8 heads of 128: over 12,564 positions 18.4
// / 18.1 us, 15,964 17.1 / 18.8, 65,536 55 / 62, 262,144 173 / 219; just above one
// unit per wave the second turn is half empty (20,064: 27.0 / 27.1 with 64 positions
// per wave there, 21.6 with 32).  40 rows of 24/4 heads of 256: 30,040 27.6 / 25.5,
// 64,040 43.8 / 48.0, 200,040 117 / 138.  At d = 64 the vector
// work decides, which is the same (no window: there 32 positions per wave).
template <int D>
bool window_takes(const jf_kv_layout& L, int32_t T, int32_t Hq, int64_t keys) {
  const int64_t units = keys / (16 * kWinNS) * L.num_kv_heads;
  return window_bytes<D>((int64_t)T * (Hq / L.num_kv_heads)) <= kWindowMax &&
         units >= (D > 128 ? 2 : 1) * (int64_t)(num_cus() / L.num_kv_heads * L.num_kv_heads) * kWinWaves * 31 / 32;
}

template <int D, bool BF16>
hipError_t launch_window_t(const jf_kv_layout& L, const jf_kv_pool_ptrs& pool, const void* q,
                           const float* lse, int32_t T, int32_t Hq, const int32_t* table,
                           int32_t prefix, float scale, float* weights, int64_t stride,
                           hipStream_t stream) {
  const auto kernel = kv8_window_weights_kernel<D, BF16>;
  const size_t lds = window_bytes<D>((int64_t)T * (Hq / L.num_kv_heads));
  if (lds > 65536) {
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel),
                                             hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
    if (e != hipSuccess) return e;
  }
  const int blocks = std::max(num_cus() / L.num_kv_heads, 1) * L.num_kv_heads;
  hipLaunchKernelGGL(kernel, dim3(blocks), dim3(kWinThreads), lds, stream,
                     static_cast<const uint8_t*>(pool.k_codes),
                     static_cast<const uint8_t*>(pool.k_meta), static_cast<const uint16_t*>(q), lse,
                     table, weights, stride, Hq, L.num_kv_heads, L.page_size,
                     shift_of(L.group_size), L.num_pages, T, prefix, std::fabs(scale) * kLog2e,
                     scale < 0.0f ? 0x80008000u : 0u);
  return hipGetLastError();
}

template <int D, bool BF16, int NS>
hipError_t launch_weights_t(const jf_kv_layout& L, const jf_kv_pool_ptrs& pool, const void* q,
                            const float* lse, int32_t T, int32_t Hq, const int32_t* table,
                            int32_t prefix, float scale, float* weights, int64_t stride,
                            hipStream_t stream) {
  const int64_t keys = (int64_t)prefix + T, per = kWWaves * 16 * NS;
  hipLaunchKernelGGL((kv8_weights_kernel<D, BF16, NS>),
                     dim3((uint32_t)((keys + per - 1) / per * L.num_kv_heads)), dim3(kWThreads), 0,
                     stream, static_cast<const uint8_t*>(pool.k_codes),
                     static_cast<const uint8_t*>(pool.k_meta), static_cast<const uint16_t*>(q), lse,
                     table, weights, stride, Hq, L.num_kv_heads, L.page_size,
                     shift_of(L.group_size), L.num_pages, T, prefix, scale * kLog2e);
  return hipGetLastError();
}
}  // namespace

hipError_t launch_kv8_weights(const jf_kv_layout& L, const jf_kv_pool_ptrs& pool, bool bf16,
                              const void* q, const float* lse, int32_t T, int32_t Hq,
                              const int32_t* block_table, int32_t prefix_len, float softmax_scale,
                              float* weights, int64_t stride, hipStream_t stream) {
  auto go = [&](auto fn) {
    return fn(L, pool, q, lse, T, Hq, block_table, prefix_len, softmax_scale, weights, stride, stream);
  };
  // What no window takes, 32 / 64 positions per wave: 64 where few columns meet many
  // positions, for fewer starts, else 32, for an even chip.  800 columns of 32/8
  // heads of 128 over 13,200 positions 40.7 / 36.0 us, 1,024 over 100,256 250 / 238;
  // 126 of 24/4 heads of 256 over 30,021 20.3 / 18.3, 600 over 60,100 93.7 / 84.9;
  // but 100 of 8/8 heads of 128 over 14,100 12.5 / 13.3, and 2,048 rows without a
  // prefix 134 / 188.  At d = 64, with few products between a wave's exponentials,
  // 32 everywhere: 512 columns of 16/2 heads over 100,064 positions 30.7 / 38.4, 896
  // of 28/4 over 30,128 28.4 / 32.1, one of 4/4 over 100,001 16.3 / 23.9.
  const int64_t keys = (int64_t)prefix_len + T;
  const bool four = (int64_t)T * (Hq / L.num_kv_heads) <= 1024 &&
                    keys / 256 * L.num_kv_heads >= num_cus() * 3 / 2;
#define JF_CASE(D_)                                                                          \
  if (L.head_dim == D_) {                                                                    \
    if constexpr (D_ > 64) {                                                                 \
      if (window_takes<D_>(L, T, Hq, keys))                                                  \
        return bf16 ? go(launch_window_t<D_, true>) : go(launch_window_t<D_, false>);        \
      if (four)                                                                              \
        return bf16 ? go(launch_weights_t<D_, true, 4>) : go(launch_weights_t<D_, false, 4>); \
    }                                                                                        \
    return bf16 ? go(launch_weights_t<D_, true, 2>) : go(launch_weights_t<D_, false, 2>);    \
  }
  JF_CASE(64)
  JF_CASE(128)
  JF_CASE(256)
#undef JF_CASE
  return hipErrorInvalidValue;
}

}  // namespace jfkv
