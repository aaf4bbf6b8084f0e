// Eviction from the 8-bit cache (format: jfkv_kv8.h) by accumulated attention
// weight: for each (request, KV head) the last `recent` positions and the
// positions of the largest weights (ties: the lowest index first), m =
// min(length, keep) in all, are moved in their order into other pages, where
// they are positions 0 .. m - 1.  Blocks there get exponents of their own,
// the least that their values allow, and a moved code changes by a power of two.
//
// HBM-bound where it is long: 4 B of weight per position (read five times, from the
// caches), and the kept codes read and written; a line of V holds four positions,
// so up to three others come along.  262,144 positions, 8 heads of 128, to 32,768:
// 91 us, of which the move takes 48 (4.5 TB/s) and six launches of the selection
// 5-8 each; four requests of up to 9,001, 4 heads of 256, to 2,000: 17 us of
// selection (one workgroup per row) and 14 of move.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "jfkv_internal.h"
#include "jfkv_kv8.h"

namespace jfkv {
namespace {

using namespace kv8;

constexpr int kBins = 2048;      // 11 bits of rank at a time
constexpr int kPerLane = 16;     // positions per lane; a wave holds 1,024 in a row
constexpr int kWavePos = 64 * kPerLane;
constexpr int kOneThreads = 1024;                           // rows of one workgroup
constexpr int kOnePos = kOneThreads * kPerLane;             // at most 16,384 positions
constexpr int kPartThreads = 512;                           // longer rows: parts of
constexpr int kPartPos = kPartThreads * kPerLane;           // 8,192 positions

// Weights in an order of unsigned integers: -inf lowest, then by value (-0 as
// +0), every NaN highest.
__device__ __forceinline__ uint32_t rank_of(float w) {
  if (w != w) return 0xffffffffu;
  if (w == 0.0f) return 0x80000000u;
  const uint32_t b = __float_as_uint(w);
  return (b & 0x80000000u) ? ~b : b | 0x80000000u;
}

// What one (request, KV head) keeps: m of n positions, the last n - cand for sure
// and `need` of the cand before them.
struct Quota {
  int n, m, cand;
  uint32_t need;
};
__device__ __forceinline__ Quota quota_of(int len, int cap, int keep, int recent) {
  const int n = min(max(len, 0), cap), m = min(n, keep), r = min(recent, n);
  return {n, m, n - r, (uint32_t)(m - r)};
}

// The ranks of the wave's positions first + 64 k + lane (0 from n on).
__device__ __forceinline__ void load_ranks(uint32_t (&rank)[kPerLane], float (&w)[kPerLane],
                                           const float* row, int first, int lane, int n) {
#pragma unroll
  for (int k = 0; k < kPerLane; ++k) {
    const int i = first + 64 * k + lane;
    w[k] = i < n ? row[i] : 0.0f;
  }
#pragma unroll
  for (int k = 0; k < kPerLane; ++k) rank[k] = rank_of(w[k]);
}

// Counts the digits (bits shift ..) of the candidates whose higher bits are
// those of limit.  Lanes that share the first such lane's digit are counted in
// one addition (equal weights would serialize the atomics).
__device__ __forceinline__ void count_digits(uint32_t* hist, const uint32_t (&rank)[kPerLane],
                                             int first, int lane, int cand, uint32_t known,
                                             uint32_t limit, int shift) {
#pragma unroll
  for (int k = 0; k < kPerLane; ++k) {
    bool on = first + 64 * k + lane < cand && (rank[k] & known) == limit;
    const uint32_t d = (rank[k] >> shift) & (kBins - 1);
    const uint64_t any = __ballot(on);
    if (!any) continue;
    const int lead = __builtin_ctzll(any);
    const uint64_t same = __ballot(on && d == (uint32_t)__builtin_amdgcn_readlane((int)d, lead));
    if (lane == lead)
      atomicAdd(&hist[d], (uint32_t)__popcll(same));
    else if (on && !(same >> lane & 1))
      atomicAdd(&hist[d], 1u);
  }
}

// The largest digit d with need <= counts of digits >= d, and what need leaves
// for d itself.  One workgroup of NT threads; scratch: NT / 64 + 2 words of LDS.
template <int NT>
__device__ __forceinline__ void find_digit(const uint32_t* hist, uint32_t need, uint32_t* scratch,
                                           uint32_t& digit, uint32_t& left) {
  constexpr int kPer = kBins / NT, kW = NT / 64;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  uint32_t c[kPer], sum = 0;
#pragma unroll
  for (int j = 0; j < kPer; ++j) sum += c[j] = hist[kBins - 1 - (tid * kPer + j)];
  uint32_t upto = sum;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const uint32_t up = __shfl_up(upto, o);
    if (lane >= o) upto += up;
  }
  if (lane == 63) scratch[wave] = upto;
  __syncthreads();
  for (int v = 0; v < wave; ++v) upto += scratch[v];
  uint32_t before = upto - sum;
  if (before < need && need <= upto) {
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
      if (before < need && need <= before + c[j]) {
        scratch[kW] = kBins - 1 - (tid * kPer + j);
        scratch[kW + 1] = need - before;
      }
      before += c[j];
    }
  }
  __syncthreads();
  digit = scratch[kW], left = scratch[kW + 1];
  __syncthreads();
}

constexpr int kShifts[3] = {21, 10, 0};
__device__ __forceinline__ uint32_t known_bits(int level) {  // before this level
  return level == 0 ? 0u : level == 1 ? 0xffe00000u : 0xfffffc00u;
}

// Which positions of the wave stay, written in order.  sure0, equal0: positions
// above and at the limit before the wave's (the recent ones count as above).
__device__ __forceinline__ void count_kept(const uint32_t (&rank)[kPerLane], int first, int lane,
                                           const Quota& t, uint32_t limit, uint32_t& sure,
                                           uint32_t& equal) {
  sure = equal = 0;
#pragma unroll
  for (int k = 0; k < kPerLane; ++k) {
    const int i = first + 64 * k + lane;
    sure += __popcll(__ballot(i < t.n && (i >= t.cand || (t.need && rank[k] > limit))));
    equal += __popcll(__ballot(t.need && i < t.cand && rank[k] == limit));
  }
}
__device__ __forceinline__ void write_kept(const uint32_t (&rank)[kPerLane],
                                           const float (&w)[kPerLane], int first, int lane,
                                           const Quota& t, uint32_t limit, uint32_t stay,
                                           uint32_t sure0, uint32_t equal0, int32_t* out,
                                           float* out_w) {
  const uint64_t below = (1ull << lane) - 1;
#pragma unroll
  for (int k = 0; k < kPerLane; ++k) {
    const int i = first + 64 * k + lane;
    const bool sure = i < t.n && (i >= t.cand || (t.need && rank[k] > limit));
    const bool same = t.need && i < t.cand && rank[k] == limit;
    const uint64_t bs = __ballot(sure), be = __ballot(same);
    const uint32_t eq = equal0 + __popcll(be & below);
    if (sure || (same && eq < stay)) {
      const uint32_t to = sure0 + __popcll(bs & below) + min(eq, stay);
      out[to] = i, out_w[to] = w[k];
    }
    sure0 += __popcll(bs), equal0 += __popcll(be);
  }
}

// Rows of at most 16,384 positions: one workgroup each, the ranks in registers
// from the first histogram to the output.
__global__ __launch_bounds__(kOneThreads) void kv8_select_kernel(
    const int32_t* __restrict__ seq_lens, const float* __restrict__ weights, int64_t stride, int cap,
    int keep, int recent, int32_t* __restrict__ kept, float* __restrict__ kept_w) {
  constexpr int kW = kOneThreads / 64;
  __shared__ uint32_t hist[kBins];
  __shared__ uint32_t scratch[kW + 2];
  __shared__ uint32_t s_sure[kW], s_equal[kW];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, first = wave * kWavePos;
  const size_t row = (size_t)blockIdx.y * gridDim.x + blockIdx.x;
  const Quota t = quota_of(seq_lens[blockIdx.y], cap, keep, recent);
  uint32_t rank[kPerLane];
  float w[kPerLane];
  load_ranks(rank, w, weights + row * stride, first, lane, t.n);
  uint32_t limit = 0, stay = t.need;
  if (t.need)
    for (int level = 0; level < 3; ++level) {
      for (int i = tid; i < kBins; i += kOneThreads) hist[i] = 0;
      __syncthreads();
      count_digits(hist, rank, first, lane, t.cand, known_bits(level), limit, kShifts[level]);
      __syncthreads();
      uint32_t d;
      find_digit<kOneThreads>(hist, stay, scratch, d, stay);
      limit |= d << kShifts[level];
    }
  uint32_t sure, equal, sure0 = 0, equal0 = 0;
  count_kept(rank, first, lane, t, limit, sure, equal);
  if (lane == 0) s_sure[wave] = sure, s_equal[wave] = equal;
  __syncthreads();
  for (int v = 0; v < wave; ++v) sure0 += s_sure[v], equal0 += s_equal[v];
  int32_t* out = kept + row * keep;
  float* out_w = kept_w + row * keep;
  write_kept(rank, w, first, lane, t, limit, stay, sure0, equal0, out, out_w);
  for (int j = t.m + tid; j < keep; j += kOneThreads) out[j] = -1, out_w[j] = 0.0f;
}

// Longer rows: parts of 8,192 positions, one launch per step.  Workspace of a
// row: three histograms, the (limit, stay) after each, and every part's counts.
struct RowState {
  uint32_t hist[3][kBins];
  uint32_t limit[3], stay[3];
};
__device__ __forceinline__ RowState* state_of(void* ws, size_t row, int parts) {
  return reinterpret_cast<RowState*>(static_cast<uint8_t*>(ws) +
                                     row * (sizeof(RowState) + sizeof(uint2) * parts));
}

__global__ void kv8_select_clear_kernel(void* ws, int parts) {
  uint32_t* h = &state_of(ws, blockIdx.x, parts)->hist[0][0];
  for (int i = threadIdx.x; i < 3 * kBins; i += blockDim.x) h[i] = 0;
}

// Level 0..2: the part's digits into the row's histogram of that level (after
// the previous level's digit was found, by every part alike).  Level 3: the
// part's counts.  Level 4: its kept positions.
template <int LEVEL>
__global__ __launch_bounds__(kPartThreads) void kv8_select_part_kernel(
    const int32_t* __restrict__ seq_lens, const float* __restrict__ weights, int64_t stride, int cap,
    int keep, int recent, int32_t* __restrict__ kept, float* __restrict__ kept_w, void* ws) {
  constexpr int kW = kPartThreads / 64;
  __shared__ uint32_t hist[LEVEL < 3 ? kBins : 1];
  __shared__ uint32_t scratch[kW + 2];
  __shared__ uint32_t s_sure[kW], s_equal[kW];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int part = blockIdx.x, parts = gridDim.x;
  const size_t row = (size_t)blockIdx.z * gridDim.y + blockIdx.y;
  const Quota t = quota_of(seq_lens[blockIdx.z], cap, keep, recent);
  RowState* st = state_of(ws, row, parts);
  uint2* counts = reinterpret_cast<uint2*>(st + 1);
  if constexpr (LEVEL == 4) {  // (this also where the row has no such part)
    for (int j = t.m + part * kPartThreads + tid; j < keep; j += parts * kPartThreads)
      kept[row * keep + j] = -1, kept_w[row * keep + j] = 0.0f;
  }
  const int base = part * kPartPos;
  if (base >= t.n) return;
  const int first = base + wave * kWavePos;
  uint32_t rank[kPerLane];
  float w[kPerLane];
  load_ranks(rank, w, weights + row * stride, first, lane, t.n);

  uint32_t limit = 0, stay = t.need;
  if constexpr (LEVEL > 0) {
    if (t.need) {
      if constexpr (LEVEL > 1 && LEVEL < 4) limit = st->limit[LEVEL - 2], stay = st->stay[LEVEL - 2];
      if constexpr (LEVEL < 4) {
        uint32_t d;
        find_digit<kPartThreads>(st->hist[LEVEL - 1], stay, scratch, d, stay);
        limit |= d << kShifts[LEVEL - 1];
        if (part == 0 && tid == 0) st->limit[LEVEL - 1] = limit, st->stay[LEVEL - 1] = stay;
      } else {
        limit = st->limit[2], stay = st->stay[2];
      }
    }
  }
  if constexpr (LEVEL < 3) {
    if (!t.need || base >= t.cand) return;
    for (int i = tid; i < kBins; i += kPartThreads) hist[i] = 0;
    __syncthreads();
    count_digits(hist, rank, first, lane, t.cand, known_bits(LEVEL), limit, kShifts[LEVEL]);
    __syncthreads();
    for (int i = tid; i < kBins; i += kPartThreads)
      if (hist[i]) atomicAdd(&st->hist[LEVEL][i], hist[i]);
  } else {
    uint32_t sure, equal;
    count_kept(rank, first, lane, t, limit, sure, equal);
    if (lane == 0) s_sure[wave] = sure, s_equal[wave] = equal;
    __syncthreads();
    if constexpr (LEVEL == 3) {
      if (tid == 0) {
        uint2 c = make_uint2(0u, 0u);
        for (int v = 0; v < kW; ++v) c.x += s_sure[v], c.y += s_equal[v];
        counts[part] = c;
      }
    } else {
      uint32_t sure0 = 0, equal0 = 0;
      for (int j = lane; j < part; j += 64) sure0 += counts[j].x, equal0 += counts[j].y;
#pragma unroll
      for (int o = 32; o; o >>= 1) sure0 += __shfl_xor(sure0, o), equal0 += __shfl_xor(equal0, o);
      for (int v = 0; v < wave; ++v) sure0 += s_sure[v], equal0 += s_equal[v];
      write_kept(rank, w, first, lane, t, limit, stay, sure0, equal0, kept + row * keep,
                 kept_w + row * keep);
    }
  }
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

  if (tid < block) {  // (a thread per token at least: the launch has min(block * D / 16, 256), block <= 128)
    int src = -1, slot = 0;
    if (tid < live) {
      const int pos = kept[((size_t)b * Hkv + h) * keep + j0 + tid];
      const int pg = src_tables[(size_t)b * max_pages + pos / P];
      slot = pos % P;
      if ((uint32_t)pg < (uint32_t)num_pages) src = pg * Hkv + h;
    }
    s_run[tid] = src, s_slot[tid] = slot;
  }
  __syncthreads();
  // The exponents are on their way along with the codes.
  int e = -126;
  if (tid < block && s_run[tid] >= 0)
    e = (int)exps[(size_t)s_run[tid] * (P / block) + (s_slot[tid] >> __builtin_ctz(block))] - 127;

  // A token without a page reads the pool's first one and counts as zeros: no
  // branch stands between the loads.
  const int dl = __builtin_ctz(D);
  uint32_t raw[NI][4];  // K: 16 dims of a token; V: four dims of four tokens
#pragma unroll
  for (int k = 0; k < NI; ++k) {
    const int i = tid + k * nthr;
    if (!is_v) {
      const int t = i >> (dl - 4), c = i & (D / 16 - 1), run = s_run[t];
      const uint4 a = *reinterpret_cast<const uint4*>(
          codes + ((size_t)max(run, 0) * P + s_slot[t]) * D + 16 * c);
      raw[k][0] = run < 0 ? 0u : a.x, raw[k][1] = run < 0 ? 0u : a.y;
      raw[k][2] = run < 0 ? 0u : a.z, raw[k][3] = run < 0 ? 0u : a.w;
    } else {
      const int r = i & (D - 1), t0 = (i >> dl) * 16 + (r % 64) / 16 * 4;
      uint4 a[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int slot = s_slot[t0 + j];
        a[j] = *reinterpret_cast<const uint4*>(
            codes + ((size_t)max(s_run[t0 + j], 0) * P + slot / 16 * 16) * D + r / 64 * 1024 +
            slot % 16 / 4 * 256 + r % 16 * 16);
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int s = 8 * (s_slot[t0 + j] % 4);
        const uint32_t m = s_run[t0 + j] < 0 ? 0u : 255u;
        raw[k][j] = ((a[j].x >> s) & m) | ((a[j].y >> s) & m) << 8 | ((a[j].z >> s) & m) << 16 |
                    ((a[j].w >> s) & m) << 24;
      }
    }
  }
  if (tid < block) s_exp[tid] = e;
  __syncthreads();

  int top = -126;  // the least exponent that the values allow
  auto look = [&](uint32_t w, int e) {
    const uint32_t a = max(max(w & 0x7fu, (w >> 8) & 0x7fu), max((w >> 16) & 0x7fu, (w >> 24) & 0x7fu));
    if (a && a != 0x7fu) top = max(top, e + exponent_for(__builtin_amdgcn_cvt_f32_fp8((int)a, 0)));
  };
#pragma unroll
  for (int k = 0; k < NI; ++k) {
    const int i = tid + k * nthr;
    const int t0 = is_v ? (i >> dl) * 16 + (i % 64) / 16 * 4 : i >> (dl - 4);
#pragma unroll
    for (int j = 0; j < 4; ++j) look(raw[k][j], s_exp[is_v ? t0 + j : t0]);
  }
#pragma unroll
  for (int o = 32; o; o >>= 1) top = max(top, __shfl_xor(top, o));
  if (lane == 0) s_max[tid >> 6] = top;
  __syncthreads();
  for (int v = 0; v < (nthr >> 6); ++v) top = max(top, s_max[v]);

  // The factor of a token's codes.  Where one is not 0 it is at most 2^17; bounded
  // for the zeros of blocks with larger exponents, as infinity would make them NaN.
  auto factor = [&](int t) { return __builtin_ldexpf(1.0f, min(s_exp[t] - top, 100)); };
#pragma unroll
  for (int k = 0; k < NI; ++k) {
    const int i = tid + k * nthr;
    uint4* const dst = reinterpret_cast<uint4*>(to) + i;
    if (!is_v) {
      const int t = i >> (dl - 4);
      if (t >= live) continue;
      const float f = factor(t);
      *dst = make_uint4(rescale4(raw[k][0], f), rescale4(raw[k][1], f), rescale4(raw[k][2], f),
                        rescale4(raw[k][3], f));
    } else {
      const int t0 = (i >> dl) * 16 + (i % 64) / 16 * 4;
      if (t0 >= live) continue;
      uint32_t c[4], o[4];
#pragma unroll
      for (int j = 0; j < 4; ++j)
        c[j] = rescale4(raw[k][j], factor(t0 + j));
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

// Parts of a row of up to cap positions, 0: one workgroup takes it whole.
int select_parts(int64_t cap) {
  return cap <= kOnePos ? 0 : (int)((cap + kPartPos - 1) / kPartPos);
}

}  // namespace

size_t kv8_evict_bytes(const jf_kv_layout& L, int32_t B, int32_t max_pages) {
  const int parts = select_parts((int64_t)max_pages * L.page_size);
  return parts ? (size_t)B * L.num_kv_heads * (sizeof(RowState) + sizeof(uint2) * parts) : 0;
}

hipError_t launch_kv8_evict(const jf_kv_layout& L, const jf_kv_pool_ptrs& pool, int32_t B,
                            const int32_t* block_tables, int32_t max_pages,
                            const int32_t* seq_lens, const float* weights, int64_t stride,
                            int32_t keep, int32_t recent, const int32_t* dst_tables,
                            int32_t dst_pages, void* ws, int32_t* kept, float* kept_w,
                            hipStream_t stream) {
  const int block = L.group_size, items = block * L.head_dim / 16;
  const int threads = std::min(items, 256);
  const int cap = max_pages * L.page_size, Hkv = L.num_kv_heads, parts = select_parts(cap);
  if (!parts) {
    hipLaunchKernelGGL(kv8_select_kernel, dim3(Hkv, B), dim3(kOneThreads), 0, stream, seq_lens,
                       weights, stride, cap, keep, recent, kept, kept_w);
  } else {
    hipLaunchKernelGGL(kv8_select_clear_kernel, dim3(Hkv * B), dim3(256), 0, stream, ws, parts);
    auto step = [&](auto kernel) {
      hipLaunchKernelGGL(kernel, dim3(parts, Hkv, B), dim3(kPartThreads), 0, stream, seq_lens,
                         weights, stride, cap, keep, recent, kept, kept_w, ws);
    };
    step(kv8_select_part_kernel<0>);
    step(kv8_select_part_kernel<1>);
    step(kv8_select_part_kernel<2>);
    step(kv8_select_part_kernel<3>);
    step(kv8_select_part_kernel<4>);
  }
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const dim3 grid(2u * (uint32_t)((std::min(keep, cap) + block - 1) / block), L.num_kv_heads, B);
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
