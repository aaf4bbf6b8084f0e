// Eviction from the 8-bit cache (format: jfkv_kv8.h) by accumulated attention
// weight: for each (request, KV head) the last `recent` positions and the
// positions of the largest weights (ties: the lowest index first), m =
// min(length, keep) in all, are moved in their order into other pages, where
// they are positions 0 .. m - 1.  Blocks there get exponents of their own,
// the least that their values allow, and a moved code changes by a power of two.
//
// HBM-bound: 4 B of weight per position, and the kept codes read and written.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "jfkv_internal.h"
#include "jfkv_kv8.h"

namespace jfkv {
namespace {

using namespace kv8;

constexpr int kSelThreads = 1024;
constexpr int kSelWaves = kSelThreads / 64;

// Weights in an order of unsigned integers: -inf lowest, then by value (-0 as
// +0), every NaN highest.
__device__ __forceinline__ uint32_t rank_of(float w) {
  if (w != w) return 0xffffffffu;
  if (w == 0.0f) return 0x80000000u;
  const uint32_t b = __float_as_uint(w);
  return (b & 0x80000000u) ? ~b : b | 0x80000000u;
}

// One workgroup per (request, KV head): radix selection of the threshold among
// the positions before the recent ones (four passes of eight bits over their
// ranks), then one pass that writes the kept positions in order.
__global__ __launch_bounds__(kSelThreads) void kv8_select_kernel(
    const int32_t* __restrict__ seq_lens, const float* __restrict__ weights, int64_t stride, int cap,
    int keep, int recent, int32_t* __restrict__ kept, float* __restrict__ kept_w) {
  __shared__ uint32_t hist[256];
  __shared__ uint32_t s_digit, s_need;
  __shared__ uint32_t s_gt[kSelWaves], s_eq[kSelWaves];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int kv = blockIdx.x, b = blockIdx.y, Hkv = gridDim.x;
  const size_t row = (size_t)b * Hkv + kv;
  const float* w = weights + row * stride;
  int32_t* out = kept + row * keep;
  float* out_w = kept_w + row * keep;

  const int n = min(max(seq_lens[b], 0), cap);
  const int m = min(n, keep), r = min(recent, n);
  const int cand = n - r;       // positions that compete
  uint32_t need = m - r;        // how many of them stay

  // threshold: the need-th largest rank; `need` becomes how many of its equals stay
  uint32_t limit = 0, known = 0;
  if (need > 0) {
    for (int shift = 24; shift >= 0; shift -= 8) {
      if (tid < 256) hist[tid] = 0;
      __syncthreads();
      for (int i = tid; i < cand; i += kSelThreads) {
        const uint32_t k = rank_of(w[i]);
        if ((k & known) == limit) atomicAdd(&hist[(k >> shift) & 255], 1u);
      }
      __syncthreads();
      if (tid == 0) {
        uint32_t left = need, d = 255;
        while (hist[d] < left) left -= hist[d--];
        s_digit = d, s_need = left;
      }
      __syncthreads();
      limit |= s_digit << shift;
      known |= 255u << shift;
      need = s_need;
      __syncthreads();
    }
  } else {
    limit = 0xffffffffu;  // (and no equal stays)
  }

  uint32_t at = 0, eq_at = 0;  // kept and equal positions so far
  for (int i0 = 0; i0 < n; i0 += kSelThreads) {
    const int i = i0 + tid;
    const float wi = i < n ? w[i] : 0.0f;
    const uint32_t k = rank_of(wi);
    const bool sure = i < n && (i >= cand || (m > r && k > limit));
    const bool equal = i < cand && m > r && k == limit;
    const uint64_t eq = __ballot(equal);
    if (lane == 0) s_eq[wave] = __popcll(eq);
    __syncthreads();
    uint32_t before = eq_at;
    for (int v = 0; v < wave; ++v) before += s_eq[v];
    const uint32_t rank = before + __popcll(eq & ((1ull << lane) - 1));
    const bool stay = sure || (equal && rank < need);
    const uint64_t gt = __ballot(stay);
    if (lane == 0) s_gt[wave] = __popcll(gt);
    __syncthreads();
    uint32_t to = at;
    for (int v = 0; v < kSelWaves; ++v) {
      if (v < wave) to += s_gt[v];
      at += s_gt[v];
      eq_at += s_eq[v];
    }
    to += __popcll(gt & ((1ull << lane) - 1));
    if (stay) out[to] = i, out_w[to] = wi;
    __syncthreads();
  }
  for (int j = m + tid; j < keep; j += kSelThreads) out[j] = -1, out_w[j] = 0.0f;
}

// One workgroup per block of destination tokens, KV head and request, for K or
// V: NI items of 16 codes per thread, as in the append.
template <int NI>
__global__ __launch_bounds__(256) void kv8_move_kernel(
    uint8_t* __restrict__ k_codes, uint8_t* __restrict__ k_exps, uint8_t* __restrict__ v_codes,
    uint8_t* __restrict__ v_exps, const int32_t* __restrict__ src_tables, int max_pages,
    const int32_t* __restrict__ dst_tables, int dst_pages, const int32_t* __restrict__ seq_lens,
    const int32_t* __restrict__ kept, int keep, int Hkv, int D, int P, int block, int num_pages) {
  __shared__ int s_run[128];   // source (page, head), -1: nothing there (zeros)
  __shared__ int s_slot[128];
  __shared__ int s_exp[128];
  __shared__ int s_max[4];
  const int tid = threadIdx.x, lane = tid & 63, nthr = blockDim.x;
  const bool is_v = blockIdx.x & 1;
  const int kb = blockIdx.x >> 1, h = blockIdx.y, b = blockIdx.z;
  const int cap = max_pages * P;
  const int m = min(min(max(seq_lens[b], 0), cap), keep);
  const int j0 = kb * block, live = min(m - j0, block);
  if (live <= 0) return;
  const int page = dst_tables[(size_t)b * dst_pages + j0 / P];
  if ((uint32_t)page >= (uint32_t)num_pages) return;
  const size_t run = (size_t)page * Hkv + h;
  uint8_t* const codes = is_v ? v_codes : k_codes;
  uint8_t* const exps = is_v ? v_exps : k_exps;
  uint8_t* const to = codes + (run * P + j0 % P) * D;

  for (int t = tid; t < block; t += nthr) {
    int src = -1, slot = 0, e = -126;
    if (t < live) {
      const int pos = kept[((size_t)b * Hkv + h) * keep + j0 + t];
      const int pg = src_tables[(size_t)b * max_pages + pos / P];
      slot = pos % P;
      if ((uint32_t)pg < (uint32_t)num_pages) {
        src = pg * Hkv + h;
        e = (int)exps[(size_t)src * (P / block) + slot / block] - 127;
      }
    }
    s_run[t] = src, s_slot[t] = slot, s_exp[t] = e;
  }
  __syncthreads();

  uint32_t raw[NI][4];  // K: 16 dims of a token; V: four dims of four tokens
  int top = -126;       // the least exponent that the values seen allow
  auto look = [&](uint32_t w, int e) {
    const uint32_t a = max(max(w & 0x7fu, (w >> 8) & 0x7fu), max((w >> 16) & 0x7fu, (w >> 24) & 0x7fu));
    if (a && a != 0x7fu) top = max(top, e + exponent_for(__builtin_amdgcn_cvt_f32_fp8((int)a, 0)));
  };
#pragma unroll
  for (int k = 0; k < NI; ++k) {
    const int i = tid + k * nthr;
#pragma unroll
    for (int j = 0; j < 4; ++j) raw[k][j] = 0u;
    if (!is_v) {
      const int t = i / (D / 16), c = i % (D / 16);
      if (s_run[t] >= 0) {
        const uint4 a = *reinterpret_cast<const uint4*>(codes + ((size_t)s_run[t] * P + s_slot[t]) * D + 16 * c);
        raw[k][0] = a.x, raw[k][1] = a.y, raw[k][2] = a.z, raw[k][3] = a.w;
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) look(raw[k][j], s_exp[t]);
    } else {
      const int r = i % D, t0 = (i / D) * 16 + (r % 64) / 16 * 4;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int t = t0 + j;
        if (s_run[t] < 0) continue;
        const int slot = s_slot[t];
        const uint4 a = *reinterpret_cast<const uint4*>(
            codes + ((size_t)s_run[t] * P + slot / 16 * 16) * D + r / 64 * 1024 +
            slot % 16 / 4 * 256 + r % 16 * 16);
        const int s = 8 * (slot % 4);
        raw[k][j] = ((a.x >> s) & 255u) | ((a.y >> s) & 255u) << 8 | ((a.z >> s) & 255u) << 16 |
                    ((a.w >> s) & 255u) << 24;
        look(raw[k][j], s_exp[t]);
      }
    }
  }
#pragma unroll
  for (int o = 32; o; o >>= 1) top = max(top, __shfl_xor(top, o));
  if (lane == 0) s_max[tid >> 6] = top;
  __syncthreads();
  for (int v = 0; v < (nthr >> 6); ++v) top = max(top, s_max[v]);

#pragma unroll
  for (int k = 0; k < NI; ++k) {
    const int i = tid + k * nthr;
    uint4* const dst = reinterpret_cast<uint4*>(to) + i;
    if (!is_v) {
      const int t = i / (D / 16);
      if (t >= live) continue;
      const float f = __builtin_ldexpf(1.0f, s_exp[t] - top);
      *dst = make_uint4(rescale4(raw[k][0], f), rescale4(raw[k][1], f), rescale4(raw[k][2], f),
                        rescale4(raw[k][3], f));
    } else {
      const int r = i % D, t0 = (i / D) * 16 + (r % 64) / 16 * 4;
      if (t0 >= live) continue;
      uint32_t c[4], o[4];
#pragma unroll
      for (int j = 0; j < 4; ++j)
        c[j] = rescale4(raw[k][j], __builtin_ldexpf(1.0f, s_exp[t0 + j] - top));
#pragma unroll
      for (int dt = 0; dt < 4; ++dt)
        o[dt] = ((c[0] >> 8 * dt) & 255u) | ((c[1] >> 8 * dt) & 255u) << 8 |
                ((c[2] >> 8 * dt) & 255u) << 16 | ((c[3] >> 8 * dt) & 255u) << 24;
      if (live - t0 < 4) {  // slots behind the last kept position stay as they are
        const uint32_t mask = 0xffffffffu >> (8 * (4 - (live - t0)));
        const uint4 a = *dst;
        o[0] = (o[0] & mask) | (a.x & ~mask), o[1] = (o[1] & mask) | (a.y & ~mask);
        o[2] = (o[2] & mask) | (a.z & ~mask), o[3] = (o[3] & mask) | (a.w & ~mask);
      }
      *dst = make_uint4(o[0], o[1], o[2], o[3]);
    }
  }
  if (tid == 0) exps[run * (P / block) + j0 % P / block] = (uint8_t)(top + 127);
}

}  // namespace

hipError_t launch_kv8_evict(const jf_kv_layout& L, const jf_kv_pool_ptrs& pool, int32_t B,
                            const int32_t* block_tables, int32_t max_pages,
                            const int32_t* seq_lens, const float* weights, int64_t stride,
                            int32_t keep, int32_t recent, const int32_t* dst_tables,
                            int32_t dst_pages, int32_t* kept, float* kept_w, hipStream_t stream) {
  const int block = L.group_size, items = block * L.head_dim / 16;
  const int threads = std::min(items, 256);
  hipLaunchKernelGGL(kv8_select_kernel, dim3(L.num_kv_heads, B), dim3(kSelThreads), 0, stream,
                     seq_lens, weights, stride, max_pages * L.page_size, keep, recent, kept, kept_w);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const dim3 grid(2u * (uint32_t)((keep + block - 1) / block), L.num_kv_heads, B);
  auto go = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, grid, dim3(threads), 0, stream, static_cast<uint8_t*>(pool.k_codes),
                       static_cast<uint8_t*>(pool.k_meta), static_cast<uint8_t*>(pool.v_codes),
                       static_cast<uint8_t*>(pool.v_meta), block_tables, max_pages, dst_tables,
                       dst_pages, seq_lens, kept, keep, L.num_kv_heads, L.head_dim, L.page_size,
                       block, L.num_pages);
    return hipGetLastError();
  };
  switch (items / threads) {
    case 1: return go(kv8_move_kernel<1>);
    case 2: return go(kv8_move_kernel<2>);
    case 4: return go(kv8_move_kernel<4>);
    default: return go(kv8_move_kernel<8>);
  }
}

}  // namespace jfkv
