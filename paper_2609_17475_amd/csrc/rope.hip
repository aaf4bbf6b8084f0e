// Rotary positions: the table of a step's angles, and the rotation of rows of
// queries and keys by it (the pairs and roundings: jfkv_rope.h).
#include <hip/hip_runtime.h>

#include <algorithm>

#include "jfkv_internal.h"
#include "jfkv_rope.h"

namespace jfkv {
namespace {

using namespace rope;

constexpr int kThreads = 256;

// (c, s) = magnitude (cos a, sin a), a = position * frequency, one pair a thread.  All
// in 64 bits, as an angle of a far position has lost its place on the circle in 32:
// the product with its rounding error (exact together), less k quarter turns
// (pi / 2 as a sum of two numbers), then the Taylor series on [-pi/4, pi/4], whose
// next terms are below 2^-37.  65,537 positions of 64 pairs: 15-16 us for 34 MB; a step's
// few rows 1.6 us, a launch.
__global__ __launch_bounds__(kThreads) void rope_table_kernel(
    const int32_t* __restrict__ positions, const float* __restrict__ freq, float* __restrict__ table,
    int half, int64_t n, float magnitude) {
  const int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  if (i >= n) return;
  const double p = positions[i / half], f = freq[i % half];
  const double a = p * f, a_lo = fma(p, f, -a);
  const double k = rint(a * 0.63661977236758134308);
  double r = fma(k, -1.5707963267948966192, a);
  r = fma(k, -6.1232339957367658e-17, r) + a_lo;
  const double z = r * r;
  double s = fma(z, -1.0 / 39916800.0, 1.0 / 362880.0);
  s = fma(z, s, -1.0 / 5040.0);
  s = fma(z, s, 1.0 / 120.0);
  s = fma(z, s, -1.0 / 6.0);
  s = fma(z * r, s, r);
  double c = fma(z, 1.0 / 479001600.0, -1.0 / 3628800.0);
  c = fma(z, c, 1.0 / 40320.0);
  c = fma(z, c, -1.0 / 720.0);
  c = fma(z, c, 1.0 / 24.0);
  c = fma(z, c, -0.5);
  c = fma(z, c, 1.0);
  const int quarter = (int)(k - 4.0 * floor(k * 0.25));
  if (quarter & 1) {
    const double t = c;
    c = -s, s = t;
  }
  const double m = quarter & 2 ? -(double)magnitude : (double)magnitude;
  reinterpret_cast<f32x2*>(table)[i] = f32x2{(float)(c * m), (float)(s * m)};
}

struct Rows {
  const uint16_t* from;
  uint16_t* to;
  int64_t from_stride, to_stride;  // elements from one token to the next
  int heads;
};

// A wave takes a run of the items of one token's heads, q's before k's; lanes 64 items on
// meet the same pairs of another head where 64 is a multiple of a head's items, and keep
// their angles then.  HBM-bound: every element read and written once, 16 bytes a lane (in
// place, only the rotated dims).  65,537 tokens of 32 + 8 heads of 128: 255 us and the
// table's 16, 5.2 TB/s, a copy's rate; 8,192 of 24 + 4 heads of 256 out of a projection's
// rows of 32 heads 51 us, 4.6 TB/s; eight tokens 3.4 us, a launch and two loads in a row.
template <int V, bool BF16, bool PAIRS>
__global__ __launch_bounds__(kThreads) void rope_rotate_kernel(
    const float* __restrict__ table, const int32_t* __restrict__ rows, int table_rows, int half,
    int D, Rows q, Rows k, int items, int segments, int per_segment, int64_t waves, float sign) {
  const int lane = threadIdx.x & 63;
  const int64_t wave = (int64_t)blockIdx.x * (kThreads / 64) + (threadIdx.x >> 6);
  if (wave >= waves) return;
  const int64_t token = wave / segments;
  const int begin = (int)(wave % segments) * per_segment;
  const int end = min(begin + per_segment, (q.heads + k.heads) * items);
  const int n_rot = half / V, head_step = 64 / items, item_step = 64 % items;
  const float* const row = table + row_of(rows, table_rows, token) * (2 * (int64_t)half);
  const uint16_t* const q_from = q.from + token * q.from_stride;
  const uint16_t* const k_from = k.from + token * k.from_stride;
  uint16_t* const q_to = q.to + token * q.to_stride;
  uint16_t* const k_to = k.to + token * k.to_stride;
  int head = (begin + lane) / items, item = (begin + lane) % items, held = -1;
  Angles<V> w;
  for (int i = begin + lane; i < end; i += 64) {
    const bool is_q = head < q.heads;
    const int64_t at = (int64_t)(is_q ? head : head - q.heads) * D;
    const uint16_t* const from = (is_q ? q_from : k_from) + at;
    uint16_t* const to = (is_q ? q_to : k_to) + at;
    int first, second;
    places<V, PAIRS>(item, n_rot, first, second);
    Elements<V> x1, x2;
    x1.load(from + first);
    x2.load(from + second);
    if (item < n_rot) {
      if (item != held) w.load(row, item, sign), held = item;
      turn<V, BF16, PAIRS>(x1, x2, w);
    }
    x1.store(to + first);
    x2.store(to + second);
    head += head_step, item += item_step;
    if (item >= items) item -= items, ++head;
  }
}

}  // namespace

hipError_t launch_rope_table(const int32_t* positions, int32_t n, const float* freq, int32_t rot,
                             float magnitude, float* table, hipStream_t stream) {
  const int64_t pairs = (int64_t)n * (rot / 2);
  hipLaunchKernelGGL(rope_table_kernel, dim3((uint32_t)((pairs + kThreads - 1) / kThreads)),
                     dim3(kThreads), 0, stream, positions, freq, table, rot / 2, pairs, magnitude);
  return hipGetLastError();
}

hipError_t launch_rope_rotate(const jf_rope& r, bool bf16, bool transpose, int32_t D,
                              const RopeRows& q, const RopeRows& k, int32_t total, hipStream_t stream) {
  const int half = r.rot_dim / 2;
  // the widest items that sizes, strides and addresses allow
  uintptr_t bits = (uintptr_t)half | (uintptr_t)((D - r.rot_dim) / 2) | 8;
  bool inplace = true;
  for (const RopeRows* x : {&q, &k})
    if (x->heads) {
      bits |= (uintptr_t)x->from_stride | (uintptr_t)x->to_stride | (uintptr_t)x->from / 2 | (uintptr_t)x->to / 2;
      inplace = inplace && x->from == x->to;
    }
  const int V = (int)(bits & -bits);
  const int items = inplace ? half / V : D / 2 / V;
  const int64_t all = (int64_t)items * (q.heads + k.heads);
  // enough waves for the chip where tokens are few
  const int64_t turns = (all + 63) / 64;
  const int64_t segments = std::max<int64_t>(1, std::min<int64_t>(turns, 4096 / total));
  const int64_t per = (turns + segments - 1) / segments * 64, waves = (int64_t)total * segments;
  auto rows = [](const RopeRows& x) {
    return Rows{static_cast<const uint16_t*>(x.from), static_cast<uint16_t*>(x.to), x.from_stride,
                x.to_stride, x.heads};
  };
  auto go = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, dim3((uint32_t)((waves + kThreads / 64 - 1) / (kThreads / 64))),
                       dim3(kThreads), 0, stream, r.table, r.rows, r.table_rows, half, D, rows(q),
                       rows(k), items, (int)segments, (int)per, waves, transpose ? -1.0f : 1.0f);
    return hipGetLastError();
  };
#define JF_CASE(V_)                                                                    \
  if (V == V_) {                                                                       \
    if (r.order == JF_ROPE_PAIRS)                                                      \
      return bf16 ? go(rope_rotate_kernel<V_, true, true>) : go(rope_rotate_kernel<V_, false, true>); \
    return bf16 ? go(rope_rotate_kernel<V_, true, false>) : go(rope_rotate_kernel<V_, false, false>); \
  }
  JF_CASE(8)
  JF_CASE(4)
  JF_CASE(2)
  JF_CASE(1)
#undef JF_CASE
  return hipErrorInvalidValue;
}

}  // namespace jfkv
