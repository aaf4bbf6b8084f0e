// Append to the 8-bit cache: rows of K and V (fp16 or bf16) become e4m3 codes
// with one exponent for each block of BT tokens of a (page, KV head); the
// format is described in jfkv_kv8.h.
//
// Per block: amax over the new rows' finite elements, e = the least exponent
// >= -126 with amax <= 448 * 2^e, raised to the block's stored exponent where
// the block already holds tokens before the first new row (start % BT != 0);
// then c = e4m3(x * 2^-e), nearest even.  If e rises, the codes of those
// earlier tokens are rescaled by 2^(e_old - e) (exact but for subnormal
// codes), so every token of a block is always read with one exponent.
//
// HBM-bound: 2 B read and 1 B written per element.  One workgroup owns one
// block of one head, of K or of V, holds its rows in registers between the
// maximum and the conversion (each row is read once), and writes 16 bytes per
// lane in the pool's own order.  262,143 rows of 8 heads of 128: 319 us, a
// copy's rate (5.05 TB/s read and written); a row of each of eight requests: 5.5 us,
// a launch and three loads that wait for one another.
#include <hip/hip_runtime.h>

#include <algorithm>

#include <type_traits>

#include "jfkv_internal.h"
#include "jfkv_kv8.h"
#include "jfkv_kv8_append_grid.h"
#include "jfkv_rope.h"

namespace jfkv {
namespace {

using namespace kv8;

// Rows of request b that the call writes: x rows r0 .. r0 + n - 1 at logical
// positions st .. st + n - 1, cut to the rows given and to the table.
struct Span {
  int r0, st, n, blocks;
};
__device__ __forceinline__ Span span_of(const int32_t* cu, const int32_t* start, int b, int total,
                                        int64_t cap, int block) {
  int r0 = min(max(cu[b], 0), total);
  int64_t n = min(max(cu[b + 1], r0), total) - r0;
  int64_t st = start[b];
  if (st < 0) {
    const int64_t skip = min(n, -st);
    r0 += (int)skip;
    n -= skip;
    st += skip;
  }
  n = max((int64_t)0, min(st + n, cap) - st);
  const int blocks = n > 0 ? (int)((st + n - 1) / block - st / block) + 1 : 0;
  return {r0, (int)st, (int)n, blocks};
}

// What the call with a rotation has besides: the rows' angles, strides of their own,
// and rows of queries.
struct Turn {
  const float* table;
  const int32_t* rows;
  int table_rows, half;
  bool pairs;
  int64_t k_stride, v_stride, q_stride;
  const uint16_t* q;
  uint16_t* q_out;
  int q_heads;
  bool together;
};
struct NoTurn {};

// 8 dims of a row of head_dim D, from dim `base` on, rotated; the partner dims are
// read from the row as well (they are another lane's, in the first-level cache).  65,535
// rows of 8 heads of 128 and 32 of queries: 313-319 us, 4.7-4.8 TB/s in and out of HBM; a row of
// each of eight requests 5.8 us, as without rotation.
template <bool BF16>
__device__ __forceinline__ void turn8(uint32_t (&raw)[4], const uint16_t* x, const float* angles,
                                      int base, int half, bool pairs) {
  using namespace rope;
  if (base >= 2 * half) return;
  if (pairs) {
    Angles<4> w;
    w.load(angles, base / 8, 1.0f);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      float y1, y2;
      turn2(half_to_float<BF16>(raw[k] & 0xffffu), half_to_float<BF16>(raw[k] >> 16), w.a[k], y1, y2);
      raw[k] = narrow2<BF16>(y1, y2);
    }
    return;
  }
  const bool second = base >= half;
  Angles<8> w;  // (the second of a pair: x2 c + x1 s = x2 c - x1 (-s))
  w.load(angles, (second ? base - half : base) / 8, second ? -1.0f : 1.0f);
  Elements<8> p;
  p.load(x + (second ? base - half : base + half));
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    float y[2], other;
#pragma unroll
    for (int i = 0; i < 2; ++i)
      turn2(half_to_float<BF16>(i ? raw[k] >> 16 : raw[k] & 0xffffu), p.template get<BF16>(2 * k + i),
            w.a[2 * k + i], y[i], other);
    raw[k] = narrow2<BF16>(y[0], y[1]);
  }
}

// The rows of queries, a token's heads by a block at a time.
template <bool BF16, bool PAIRS>
__device__ __forceinline__ void turn_queries(const Turn& r, int D, int unit, int units, int h, int heads,
                                             int total) {
  using namespace rope;
  const int items = D / 16, n_rot = r.half / 8;
  const append::Tokens turn_of = append::tokens_of(r.together, unit, units, h, heads, total);
  for (int64_t t = turn_of.first; t < turn_of.end; t += turn_of.step) {
    const float* const angles = r.table + row_of(r.rows, r.table_rows, t) * (2 * (int64_t)r.half);
    for (int i = threadIdx.x; i < r.q_heads * items; i += blockDim.x) {
      const int item = i % items, at = i / items * D;
      int first, second;
      places<8, PAIRS>(item, n_rot, first, second);
      const uint16_t* const x = r.q + t * r.q_stride + at;
      uint16_t* const y = r.q_out + t * ((int64_t)r.q_heads * D) + at;
      Elements<8> x1, x2;
      x1.load(x + first);
      x2.load(x + second);
      if (item < n_rot) {
        Angles<8> w;
        w.load(angles, item, 1.0f);
        turn<8, BF16, PAIRS>(x1, x2, w);
      }
      x1.store(y + first);
      x2.store(y + second);
    }
  }
}

// NI items of 16 elements per thread: for K 16 dims of a token, for V 4 dims
// of 4 tokens (the 16 bytes that lie together in the pool).  ROPE: K's rows are
// rotated on the way, rounded to their type as a rotation by itself would leave
// them, so that both ways write the same cache; blocks of z = 2 rotate queries.
template <int NI, bool BF16, bool ROPE>
__global__ __launch_bounds__(256) void kv8_append_kernel(
    uint8_t* __restrict__ k_codes, uint8_t* __restrict__ k_exps, uint8_t* __restrict__ v_codes,
    uint8_t* __restrict__ v_exps, const uint16_t* __restrict__ k_new,
    const uint16_t* __restrict__ v_new, const int32_t* __restrict__ cu,
    const int32_t* __restrict__ start, const int32_t* __restrict__ block_tables, int B, int Hkv,
    int D, int P, int block, int num_pages, int max_pages, int total,
    std::conditional_t<ROPE, Turn, NoTurn> rope) {
  constexpr uint32_t kInf = BF16 ? 0x7f80u : 0x7c00u;  // magnitudes from here on are not finite
  __shared__ uint32_t s_max[4];
  const int tid = threadIdx.x, lane = tid & 63, nthr = blockDim.x;
  int unit = blockIdx.x, h = blockIdx.y, part = blockIdx.z;
  const int64_t cap = (int64_t)max_pages * P;
  if constexpr (ROPE) {
    if (rope.together) {
      const append::Place at = append::place_of(unit, h, part, gridDim.x, gridDim.y, gridDim.z);
      unit = at.unit, h = at.head, part = at.part;
    }
    if (part == 2) {
      if (rope.pairs)
        turn_queries<BF16, true>(rope, D, unit, gridDim.x, h, gridDim.y, total);
      else
        turn_queries<BF16, false>(rope, D, unit, gridDim.x, h, gridDim.y, total);
      return;
    }
  }
  const bool is_v = part != 0;

  // ---- the request and block of this unit: every wave scans the block counts
  int u = unit, b = 0;
  Span sp;
  if (B == 1) {
    sp = span_of(cu, start, 0, total, cap, block);
    if (u >= sp.blocks) return;
  } else {
    bool found = false;
    for (int b0 = 0; b0 < B && !found; b0 += 64) {
      const int bb = b0 + lane;
      const int cnt = bb < B ? span_of(cu, start, bb, total, cap, block).blocks : 0;
      int64_t sum = cnt;
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) {
        const int64_t up = __shfl_up(sum, o);
        if (lane >= o) sum += up;
      }
      const uint64_t hit = __ballot(u < sum);
      if (hit) {
        const int l = __builtin_ctzll(hit);
        b = b0 + l;
        u -= (int)(__shfl(sum, l) - __shfl(cnt, l));
        found = true;
      } else {
        u -= (int)__shfl(sum, 63);
      }
    }
    if (!found) return;
    sp = span_of(cu, start, b, total, cap, block);
  }
  const int kb = sp.st / block + u;                            // block of the request
  const int64_t pos0 = (int64_t)kb * block;                    // its first position
  const int lo = (int)max((int64_t)0, sp.st - pos0);           // new rows at slots lo ..
  const int hi = (int)min((int64_t)block, sp.st + (int64_t)sp.n - pos0);  // .. hi - 1 of it
  const int page = block_tables[(size_t)b * max_pages + pos0 / P];
  if ((uint32_t)page >= (uint32_t)num_pages) return;
  const int slot0 = (int)(pos0 % P);
  const size_t run = (size_t)page * Hkv + h;
  uint8_t* const codes = (is_v ? v_codes : k_codes) + (run * P + slot0) * D;
  uint8_t* const exps = (is_v ? v_exps : k_exps) + run * (P / block) + slot0 / block;
  const uint16_t* const x = is_v ? v_new : k_new;
  const int e_old = lo > 0 ? (int)*exps - 127 : -126;

  // element offset of slot s's row (in range for lo <= s < hi)
  const int64_t row_base = sp.r0 + pos0 - sp.st;
  size_t row_stride = (size_t)Hkv * D;
  if constexpr (ROPE) row_stride = is_v ? rope.v_stride : rope.k_stride;
  const uint16_t* const xh = x + (size_t)h * D;

  // ---- load, and the largest finite magnitude as 16-bit patterns
  uint32_t raw[NI][8];
  uint32_t top = 0;
#pragma unroll
  for (int k = 0; k < NI; ++k) {
    const int i = tid + k * nthr;
#pragma unroll
    for (int j = 0; j < 8; ++j) raw[k][j] = 0u;
    if (!is_v) {
      const int t = i / (D / 16), c = i % (D / 16);
      if (t >= lo && t < hi) {
        const uint4* src = reinterpret_cast<const uint4*>(xh + (row_base + t) * row_stride + 16 * c);
        const uint4 a = src[0], d = src[1];
        raw[k][0] = a.x, raw[k][1] = a.y, raw[k][2] = a.z, raw[k][3] = a.w;
        raw[k][4] = d.x, raw[k][5] = d.y, raw[k][6] = d.z, raw[k][7] = d.w;
        if constexpr (ROPE) {
          const uint16_t* const row = xh + (row_base + t) * row_stride;
          const float* const angles =
              rope.table + rope::row_of(rope.rows, rope.table_rows, row_base + t) * (2 * (int64_t)rope.half);
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            uint32_t part[4] = {raw[k][4 * j], raw[k][4 * j + 1], raw[k][4 * j + 2], raw[k][4 * j + 3]};
            turn8<BF16>(part, row, angles, 16 * c + 8 * j, rope.half, rope.pairs);
#pragma unroll
            for (int i = 0; i < 4; ++i) raw[k][4 * j + i] = part[i];
          }
        }
      }
    } else {
      const int r = i % D, t0 = (i / D) * 16 + (r % 64) / 16 * 4, dim = r / 64 * 64 + (r % 16) * 4;
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (t0 + j >= lo && t0 + j < hi) {
          const uint2 a = *reinterpret_cast<const uint2*>(xh + (row_base + t0 + j) * row_stride + dim);
          raw[k][2 * j] = a.x, raw[k][2 * j + 1] = a.y;
        }
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const uint32_t l = raw[k][j] & 0x7fffu, m = (raw[k][j] >> 16) & 0x7fffu;
      top = max(top, max(l < kInf ? l : 0u, m < kInf ? m : 0u));
    }
  }
#pragma unroll
  for (int o = 32; o; o >>= 1) top = max(top, (uint32_t)__shfl_xor((int)top, o));
  if (lane == 0) s_max[tid >> 6] = top;
  __syncthreads();
  for (int w = 0; w < (nthr >> 6); ++w) top = max(top, s_max[w]);

  const int e = max(exponent_for(half_to_float<BF16>(top)), e_old);
  const float inv = power2(-e);
  const bool grow = lo > 0 && e != e_old;
  const float shrink = power2(e_old - e);

  // ---- convert and store
#pragma unroll
  for (int k = 0; k < NI; ++k) {
    const int i = tid + k * nthr;
    uint4* const dst = reinterpret_cast<uint4*>(codes) + i;
    if (!is_v) {
      const int t = i / (D / 16);
      if (t >= lo && t < hi) {
        uint32_t o[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const uint32_t a = raw[k][2 * j], c = raw[k][2 * j + 1];
          o[j] = encode2<false>(half_to_float<BF16>(a & 0xffffu) * inv,
                                half_to_float<BF16>(a >> 16) * inv, 0u);
          o[j] = encode2<true>(half_to_float<BF16>(c & 0xffffu) * inv,
                               half_to_float<BF16>(c >> 16) * inv, o[j]);
        }
        *dst = make_uint4(o[0], o[1], o[2], o[3]);
      } else if (t < lo && grow) {
        const uint4 a = *dst;
        *dst = make_uint4(rescale4(a.x, shrink), rescale4(a.y, shrink), rescale4(a.z, shrink),
                          rescale4(a.w, shrink));
      }
    } else {
      const int r = i % D, t0 = (i / D) * 16 + (r % 64) / 16 * 4;
      const int first = max(lo - t0, 0), last = min(hi - t0, 4);  // new tokens of the four
      if (first < last || (grow && t0 < lo)) {
        uint32_t o[4];
#pragma unroll
        for (int dt = 0; dt < 4; ++dt) {
          float v[4];
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const uint32_t a = raw[k][2 * j + dt / 2];
            v[j] = half_to_float<BF16>(dt % 2 ? a >> 16 : a & 0xffffu) * inv;
          }
          o[dt] = encode2<true>(v[2], v[3], encode2<false>(v[0], v[1], 0u));
        }
        if (first > 0 || last < 4) {  // the others of the four keep what they hold
          const uint32_t fresh = first < last ? (0xffffffffu >> (8 * (4 - (last - first)))) << (8 * first) : 0u;
          const int olds = min(max(lo - t0, 0), 4);
          const uint32_t before = olds ? 0xffffffffu >> (8 * (4 - olds)) : 0u;
          const uint4 a = *dst;
          const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
          for (int dt = 0; dt < 4; ++dt) {
            uint32_t held = w[dt];
            if (grow) held = (rescale4(held, shrink) & before) | (held & ~before);
            o[dt] = (o[dt] & fresh) | (held & ~fresh);
          }
        }
        *dst = make_uint4(o[0], o[1], o[2], o[3]);
      }
    }
  }
  if (tid == 0) *exps = (uint8_t)(e + 127);
}

}  // namespace

namespace {
template <bool ROPE, class T>
hipError_t launch_append(const jf_kv_layout& L, const jf_kv_pool_ptrs& pool, bool bf16,
                         const void* k_new, const void* v_new, const int32_t* cu_tok,
                         const int32_t* start_pos, const int32_t* block_tables, int32_t B,
                         int32_t max_pages, int32_t total_tok, const T& rope, int64_t units, int parts,
                         hipStream_t stream) {
  const int block = L.group_size, items = block * L.head_dim / 16;
  const int threads = std::min(items, 256);
  const dim3 grid((uint32_t)units, L.num_kv_heads, parts);
  auto go = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, grid, dim3(threads), 0, stream, static_cast<uint8_t*>(pool.k_codes),
                       static_cast<uint8_t*>(pool.k_meta), static_cast<uint8_t*>(pool.v_codes),
                       static_cast<uint8_t*>(pool.v_meta), static_cast<const uint16_t*>(k_new),
                       static_cast<const uint16_t*>(v_new), cu_tok, start_pos, block_tables, B,
                       L.num_kv_heads, L.head_dim, L.page_size, block, L.num_pages, max_pages,
                       total_tok, rope);
    return hipGetLastError();
  };
  switch (items / threads) {
    case 1: return bf16 ? go(kv8_append_kernel<1, true, ROPE>) : go(kv8_append_kernel<1, false, ROPE>);
    case 2: return bf16 ? go(kv8_append_kernel<2, true, ROPE>) : go(kv8_append_kernel<2, false, ROPE>);
    case 4: return bf16 ? go(kv8_append_kernel<4, true, ROPE>) : go(kv8_append_kernel<4, false, ROPE>);
    default: return bf16 ? go(kv8_append_kernel<8, true, ROPE>) : go(kv8_append_kernel<8, false, ROPE>);
  }
}
}  // namespace

hipError_t launch_kv8_append(const jf_kv_layout& L, const jf_kv_pool_ptrs& pool, bool bf16,
                             const void* k_new, const void* v_new, const int32_t* cu_tok,
                             const int32_t* start_pos, const int32_t* block_tables, int32_t B,
                             int32_t max_pages, int32_t total_tok, hipStream_t stream) {
  return launch_append<false>(L, pool, bf16, k_new, v_new, cu_tok, start_pos, block_tables, B,
                              max_pages, total_tok, NoTurn{}, append::units_of(total_tok, B, L.group_size), 2,
                              stream);
}

hipError_t launch_kv8_rope_append(const jf_kv_layout& L, const jf_kv_pool_ptrs& pool, bool bf16,
                                  const jf_rope& r, const void* k_new, int64_t k_stride,
                                  const void* v_new, int64_t v_stride, const void* q, int64_t q_stride,
                                  void* q_out, int32_t Hq, const int32_t* cu_tok,
                                  const int32_t* start_pos, const int32_t* block_tables, int32_t B,
                                  int32_t max_pages, int32_t total_tok, hipStream_t stream) {
  const int parts = q ? 3 : 2;
  const append::Grid grid = append::grid_of(total_tok, B, L.group_size, r.rot_dim, L.num_kv_heads, parts);
  const Turn turn{r.table, r.rows, r.table_rows, r.rot_dim / 2, r.order == JF_ROPE_PAIRS,
                  k_stride, v_stride, q_stride, static_cast<const uint16_t*>(q),
                  static_cast<uint16_t*>(q_out), Hq, grid.together};
  return launch_append<true>(L, pool, bf16, k_new, v_new, cu_tok, start_pos, block_tables, B,
                             max_pages, total_tok, turn, grid.units, parts, stream);
}

}  // namespace jfkv
