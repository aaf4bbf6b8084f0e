// Device helpers of the rotary positions: one item of a head's row at a time.
//
// A head of D dims has R / 2 pairs of rotated dims and D - R dims that are only
// copied.  An item is V pairs, or 2 V copied dims: items 0 .. R / 2 / V - 1 rotate,
// the others copy.
//   (y1, y2) = (x1 c - x2 s, x2 c + x1 s)
// with every product and sum rounded in fp32 by itself (no fused products: an
// elementary form in fp32 then gives the same bits), and the result once to its type.
#pragma once

#include "jfkv_kv8.h"

namespace jfkv {
namespace rope {

using kv8::f32x2;

// V 16-bit elements.
template <int V>
struct Elements {
  uint32_t w[V / 2];
  __device__ __forceinline__ void load(const uint16_t* p) {
    __builtin_memcpy(w, __builtin_assume_aligned(p, 2 * V), 2 * V);
  }
  __device__ __forceinline__ void store(uint16_t* p) const {
    __builtin_memcpy(__builtin_assume_aligned(p, 2 * V), w, 2 * V);
  }
  template <bool BF16>
  __device__ __forceinline__ float get(int i) const {
    return kv8::half_to_float<BF16>(i % 2 ? w[i / 2] >> 16 : w[i / 2] & 0xffffu);
  }
  template <bool BF16>
  __device__ __forceinline__ void set(int i, float a, float b) { w[i / 2] = kv8::narrow2<BF16>(a, b); }
};
template <>
struct Elements<1> {
  uint16_t w;
  __device__ __forceinline__ void load(const uint16_t* p) { w = *p; }
  __device__ __forceinline__ void store(uint16_t* p) const { *p = w; }
  template <bool BF16>
  __device__ __forceinline__ float get(int) const { return kv8::half_to_float<BF16>(w); }
};

__device__ __forceinline__ void turn2(float x1, float x2, f32x2 a, float& y1, float& y2) {
#pragma clang fp contract(off)
  y1 = x1 * a.x - x2 * a.y;
  y2 = x2 * a.x + x1 * a.y;
}

// (c, s) of the V pairs of item i of a table row; sign -1 turns back.
template <int V>
struct Angles {
  f32x2 a[V];
  __device__ __forceinline__ void load(const float* row, int i, float sign) {
    __builtin_memcpy(a, __builtin_assume_aligned(row + 2 * V * i, 8), sizeof(a));
#pragma unroll
    for (int k = 0; k < V; ++k) a[k].y *= sign;
  }
};

// The two runs of V dims that item i reads and writes.
template <int V, bool PAIRS>
__device__ __forceinline__ void places(int i, int n_rot, int& first, int& second) {
  if (PAIRS || i >= n_rot) {
    first = 2 * V * i, second = first + V;
  } else {
    first = V * i, second = first + V * n_rot;
  }
}

template <int V, bool BF16, bool PAIRS>
__device__ __forceinline__ void turn(Elements<V>& p, Elements<V>& q, const Angles<V>& w) {
  if constexpr (V == 1) {  // (a pair's two elements, wherever they lie)
    float y1, y2;
    turn2(p.template get<BF16>(0), q.template get<BF16>(0), w.a[0], y1, y2);
    const uint32_t y = kv8::narrow2<BF16>(y1, y2);
    p.w = (uint16_t)y, q.w = (uint16_t)(y >> 16);
  } else if constexpr (PAIRS) {
#pragma unroll
    for (int k = 0; k < V; ++k) {
      Elements<V>& e = k < V / 2 ? p : q;
      const int at = 2 * k % V;
      float y1, y2;
      turn2(e.template get<BF16>(at), e.template get<BF16>(at + 1), w.a[k], y1, y2);
      e.template set<BF16>(at, y1, y2);
    }
  } else {
#pragma unroll
    for (int k = 0; k < V; k += 2) {
      float a1, a2, b1, b2;
      turn2(p.template get<BF16>(k), q.template get<BF16>(k), w.a[k], a1, b1);
      turn2(p.template get<BF16>(k + 1), q.template get<BF16>(k + 1), w.a[k + 1], a2, b2);
      p.template set<BF16>(k, a1, a2);
      q.template set<BF16>(k, b1, b2);
    }
  }
}

// The table row of token i (an index outside the table is cut to it).
__device__ __forceinline__ int64_t row_of(const int32_t* rows, int table_rows, int64_t i) {
  return rows ? min(max(rows[i], 0), table_rows - 1) : i;
}

}  // namespace rope
}  // namespace jfkv
