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

#include "jfkv_internal.h"
#include "jfkv_kv8.h"

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

// NI items of 16 elements per thread: for K 16 dims of a token, for V 4 dims
// of 4 tokens (the 16 bytes that lie together in the pool).
template <int NI, bool BF16>
__global__ __launch_bounds__(256) void kv8_append_kernel(
    uint8_t* __restrict__ k_codes, uint8_t* __restrict__ k_exps, uint8_t* __restrict__ v_codes,
    uint8_t* __restrict__ v_exps, const uint16_t* __restrict__ k_new,
    const uint16_t* __restrict__ v_new, const int32_t* __restrict__ cu,
    const int32_t* __restrict__ start, const int32_t* __restrict__ block_tables, int B, int Hkv,
    int D, int P, int block, int num_pages, int max_pages, int total) {
  constexpr uint32_t kInf = BF16 ? 0x7f80u : 0x7c00u;  // magnitudes from here on are not finite
  __shared__ uint32_t s_max[4];
  const int tid = threadIdx.x, lane = tid & 63, nthr = blockDim.x;
  const int h = blockIdx.y;
  const bool is_v = blockIdx.z != 0;
  const int64_t cap = (int64_t)max_pages * P;

  // ---- the request and block of this unit: every wave scans the block counts
  int u = blockIdx.x, b = 0;
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
  const size_t row_stride = (size_t)Hkv * D;
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

hipError_t launch_kv8_append(const jf_kv_layout& L, const jf_kv_pool_ptrs& pool, bool bf16,
                             const void* k_new, const void* v_new, const int32_t* cu_tok,
                             const int32_t* start_pos, const int32_t* block_tables, int32_t B,
                             int32_t max_pages, int32_t total_tok, hipStream_t stream) {
  const int block = L.group_size, items = block * L.head_dim / 16;
  const int threads = std::min(items, 256);
  // blocks that total_tok rows of B requests can touch: one per row at most,
  // and whole blocks plus two partial ones per request
  const int64_t units = std::min<int64_t>(total_tok, total_tok / block + 2 * (int64_t)B);
  const dim3 grid((uint32_t)units, L.num_kv_heads, 2);
  auto go = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, grid, dim3(threads), 0, stream, static_cast<uint8_t*>(pool.k_codes),
                       static_cast<uint8_t*>(pool.k_meta), static_cast<uint8_t*>(pool.v_codes),
                       static_cast<uint8_t*>(pool.v_meta), static_cast<const uint16_t*>(k_new),
                       static_cast<const uint16_t*>(v_new), cu_tok, start_pos, block_tables, B,
                       L.num_kv_heads, L.head_dim, L.page_size, block, L.num_pages, max_pages,
                       total_tok);
    return hipGetLastError();
  };
  switch (items / threads) {
    case 1: return bf16 ? go(kv8_append_kernel<1, true>) : go(kv8_append_kernel<1, false>);
    case 2: return bf16 ? go(kv8_append_kernel<2, true>) : go(kv8_append_kernel<2, false>);
    case 4: return bf16 ? go(kv8_append_kernel<4, true>) : go(kv8_append_kernel<4, false>);
    default: return bf16 ? go(kv8_append_kernel<8, true>) : go(kv8_append_kernel<8, false>);
  }
}

}  // namespace jfkv
