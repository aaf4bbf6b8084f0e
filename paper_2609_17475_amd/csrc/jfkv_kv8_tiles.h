// A walk over tiles of 64 positions (format: jfkv_kv8.h) of one KV head: a block of eight
// waves, each with column sets of its own, all of which see the same positions but for
// what `Sees` hides.  It is the chunk attention's (kv8_prefill.hip says what bounds it)
// with an order of its own within a turn; that kernel, whose causal masks end each
// block elsewhere, keeps its own text: with this one it took 2-7 % longer.
//
// A turn of 64 positions, 256 columns and d = 128 takes some 4,900 cycles: the products
// 1,700 (1,024 of matrix cores, 1,024 of LDS reads for four waves), the softmax 1,800
// (32 exponentials at a quarter of the rate and some 100 vector instructions), the next
// tiles' way into LDS 700-900.  Two waves of a SIMD take products and softmax in turns.
// 1,024 columns over 65,536 positions: 300-322 us, 850-920 TFLOP/s.
#pragma once

#include <type_traits>

#include "jfkv_kv8.h"

namespace jfkv {
namespace kv8 {
namespace tiles {

#define JF_INLINE __attribute__((always_inline))

constexpr int kTile = 64;        // positions of a tile (in one page)
constexpr int kWaves = 8;
constexpr int kThreads = 64 * kWaves;
constexpr uint32_t kZeroExp = 1;  // the exponent byte of a block of zeros
constexpr float kLog2e = 1.44269504088896340736f;

// The query row of (row, head) as B operands: dims 64 c + 16 g + 8 j ..
template <int C, bool BF16>
__device__ __forceinline__ void load_q(u32x4 (&qf)[C][2], const uint16_t* qp, int g, uint32_t flip) {
#pragma unroll
  for (int c = 0; c < C; ++c)
#pragma unroll
    for (int j = 0; j < 2; ++j)
      qf[c][j] = *reinterpret_cast<const u32x4*>(qp + 64 * c + 16 * g + 8 * j) ^ flip;
}

// Tiles j0 .. j1 - 1 of a KV head for the columns of the block's waves: NC sets of 16 a
// wave, whose queries are qf and which see the positions below see (`least`: the least
// of the wave's).  L: positions that are written.  A tile's K and V codes are fetched
// into registers two tiles ahead, widened once for the block and laid into LDS as the
// matrix operands that all waves read.  acc (in units of 2^e_ref), m and l (log2 units)
// grow.  Waves that are not active only carry.  table: a pointer to int32.
template <int D, bool BF16, int NC, class Table, class Sees>
__device__ __forceinline__ void walk_tiles(
    const uint8_t* k_codes, const uint8_t* k_exps,
    const uint8_t* v_codes, const uint8_t* v_exps,
    int tid, Table table, int Hkv, int kv, int P, int block_shift, int num_pages, int L,
    int j0, int j1, float scale_log2, const u32x4 (&qf)[NC][D / 64][2], const Sees& sees,
    bool active, u32x4* lds,
    f32x4 (&acc)[NC][D / 64][4], float (&m)[NC], float (&l)[NC], int& e_ref, int& e_top) {
  constexpr int C = D / 64, kTileSize = 8 * D;
  const int lane = tid & 63, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  // Two tiles of K and V each, in the order V1 K0 V0 K1: a turn's operands, V of one tile
  // and K of the next, follow one another.
  auto tile_k = [&](int j) JF_INLINE { return lds + (j & 1 ? 3 : 1) * kTileSize; };
  auto tile_v = [&](int j) JF_INLINE { return lds + (j & 1 ? 0 : 2) * kTileSize; };
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
  // else's.  (Its values are cleared by a mask on every tile: a branch costs more.)
  auto held = [&](int pid) JF_INLINE { return (uint32_t)pid < (uint32_t)num_pages; };
  // (pages times heads are below 2^31)
  auto run_of = [&](int pid) JF_INLINE { return (uint32_t)(held(pid) ? pid : 0) * (uint32_t)Hkv + (uint32_t)kv; };
  auto place = [&](int slot0, int pid) JF_INLINE {
    return ((uint64_t)run_of(pid) * (uint32_t)P + (uint32_t)slot0) * D;
  };
  const uint32_t k_off = (tid % kOf / D * 16 + (lane & 15)) * D + tid % D / 64 * 64 + (lane >> 4) * 16;
  auto fetch_k = [&](int slot0, int pid) JF_INLINE {
    const uint8_t* kp = k_codes + place(slot0, pid);
#pragma unroll
    for (int k = 0; k < kPieces; ++k)
      k_stage[k] = *reinterpret_cast<const u32x4*>(kp + k_off + k * (kThreads / D) * 16 * D);
    const uint8_t* ep = (lane & 4) ? v_exps : k_exps;
    exps_next = ep[(uint64_t)run_of(pid) * (uint32_t)(P >> block_shift) +
                   (uint32_t)((slot0 + 16 * (lane & 3)) >> block_shift)];
  };
  auto fetch_v = [&](int slot0, int pid) JF_INLINE {
    const uint8_t* vp = v_codes + place(slot0, pid);
#pragma unroll
    for (int k = 0; k < kPieces; ++k)
      v_stage[k] = *reinterpret_cast<const u32x4*>(vp + (tid % kOf + k * kThreads) * 16);
  };
  auto deposit_k = [&](int j) JF_INLINE {
    if (kOf < kThreads && tid >= kOf) return;
#pragma unroll
    for (int k = 0; k < kPieces; ++k) {
      const int i = tid + k * kThreads;
      // [16 positions][64 dims][half][lane]
      u32x4* to = tile_k(j) + i / 64 * 128 + i % 64;
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
      u32x2* to = reinterpret_cast<u32x2*>(tile_v(j) + (i / D / 2 * C + i % D / 64) * 256 + i % 64) + i / D % 2;
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

  auto softmax = [&](int j, bool on) JF_INLINE {
    const int pos0 = j * kTile;
    if (!on || sees.hides_some(pos0)) {
#pragma unroll
      for (int t = 0; t < 4; ++t) {
#pragma unroll
        for (int cs = 0; cs < NC; ++cs)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (!on || sees.hides(cs, pos0 + 16 * t + 4 * g + i)) s[t][cs][i] = -INFINITY;
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

  // The products of turn j: the values of tile j - 1, then the scores of tile j.  Their
  // operands are one run in LDS, each read kAhead before its products, so that a turn
  // waits for the first of them only once.  (The barriers keep the compiler from reading
  // all of them at once, which spills; with two sets of columns or d = 256 eight ahead
  // spill too.)
  constexpr int kAhead = NC == 1 && D <= 128 ? 8 : 4, kV = 8 * C, kAll = 16 * C;
  auto products = [&](int j) JF_INLINE {
    const u32x4* const from = lds + (j & 1 ? 2 : 0) * kTileSize + lane;
    // the scores' operands with the four groups of 16 positions in turn, so that no
    // product waits for the one before it
    auto operand = [&](int p) JF_INLINE {
      const int k = p - kV;
      return from[64 * (p < kV ? p : kV + k % 4 * (2 * C) + k / 4)];
    };
    u32x4 ring[kAhead];
    if (j > j0 && !apart) {
#pragma unroll
      for (int p = 0; p < kAhead; ++p) ring[p] = operand(p);
#pragma unroll
      for (int p = 0; p < kV; ++p) {
        const int t2 = p / (4 * C), c = p / 4 % C, dt = p % 4;
        const u32x4 a = ring[p % kAhead];
        ring[p % kAhead] = operand(p + kAhead);  // (after the last tile: what is there)
#pragma unroll
        for (int cs = 0; cs < NC; ++cs) {
          const u32x4 b = {pf[t2][cs][0], pf[t2][cs][1], pf[t2][cs][2], pf[t2][cs][3]};
          acc[cs][c][dt] = mma<false>(a, b, acc[cs][c][dt]);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    } else {
      if (j > j0) {
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          rescale(reference_step(e_ref, split_e[t]));
          e_ref = split_e[t];
#pragma unroll
          for (int p = 0; p < 4 * C; ++p) {
            const u32x4 a = operand(t / 2 * 4 * C + p);
#pragma unroll
            for (int cs = 0; cs < NC; ++cs) {
              const u32x4 b = t % 2 ? u32x4{0u, 0u, pf[t / 2][cs][2], pf[t / 2][cs][3]}
                                    : u32x4{pf[t / 2][cs][0], pf[t / 2][cs][1], 0u, 0u};
              acc[cs][p / 4][p % 4] = mma<false>(a, b, acc[cs][p / 4][p % 4]);
            }
            __builtin_amdgcn_sched_barrier(0);
          }
        }
      }
#pragma unroll
      for (int p = 0; p < kAhead; ++p) ring[p] = operand(kV + p);
    }
    if (j == j1) return;
#pragma unroll
    for (int t = 0; t < 4; ++t) {
#pragma unroll
      for (int cs = 0; cs < NC; ++cs) s[t][cs] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
      // (not 0, so that a hidden score times it stays -inf)
      f[t] = fmaxf(scale_log2 * power2(__builtin_amdgcn_readlane((int)exps, t) - 127), 1e-37f);
      ev[t] = __builtin_amdgcn_readlane((int)exps, 4 + t) - 127;
    }
#pragma unroll
    for (int p = kV; p < kAll; ++p) {
      const int t = (p - kV) % 4, c = (p - kV) / 8, half = (p - kV) / 4 % 2;
      const u32x4 a = ring[p % kAhead];
      if (p + kAhead < kAll) ring[p % kAhead] = operand(p + kAhead);
#pragma unroll
      for (int cs = 0; cs < NC; ++cs) s[t][cs] = mma<BF16>(a, qf[cs][c][half], s[t][cs]);
      __builtin_amdgcn_sched_barrier(0);
    }
  };

  // ---- Turn j forms the scores of tile j and the value products of tile j - 1.
  // Waves w and w + 4 share a SIMD: the first do their matrix products at once and
  // the softmax after them, the second the other way round, so that one's matrix
  // products meet the other's vector work; both carry the next tiles last (between the
  // two, as the chunk attention does: 1,024 columns over 65,536 positions 361 us against
  // 322, 256 columns 117 against 108).  At d = 64, where the vector work is the most, all
  // do the same.  (Two loops, as one loop with both orders spills; every wave passes
  // j1 - j0 + 1 barriers in either.)
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
    for (int j = j0; j <= j1; ++j) {
      __syncthreads();  // K of tile j and V of tile j - 1 are in LDS
      const int pid_n = page_of(at);
      uint32_t exps_1;  // of tile j + 1
      // (Without a condition, past the last tile too, where it carries what nobody reads:
      // the compiler then knows how many loads are on the way, and waits for the one
      // that it needs and not for all.  Taken before the next are fetched, exps_1 needs
      // no copy that would wait at the end of the turn.)
      auto transport = [&]() JF_INLINE {
        deposit_v(j, held(pid[1]) ? 0xffffffffu : 0u);
        fetch_v(slot[2], pid[2]);
        deposit_k(j + 1);
        exps_1 = held(pid[2]) ? exps_next : kZeroExp;
        asm volatile("" : "+v"(exps_1));
        __builtin_amdgcn_sched_barrier(0);
        fetch_k(slot[3], pid[3]);
      };
      if constexpr (late) {
        if (active && j > j0) softmax(j - 1, (uint32_t)pid[0] < (uint32_t)num_pages);
      }
      __builtin_amdgcn_s_setprio(1);
      if (active) products(j);
      __builtin_amdgcn_s_setprio(0);
      if constexpr (!late) {
        if (active && j < j1) softmax(j, (uint32_t)pid[1] < (uint32_t)num_pages);
      }
      transport();
      exps = exps_1;
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
}

}  // namespace tiles
}  // namespace kv8
}  // namespace jfkv
