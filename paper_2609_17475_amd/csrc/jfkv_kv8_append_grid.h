// How the blocks of an append to the 8-bit cache (kv8_append.hip) share its work: units
// (blocks of tokens) x KV heads x parts (K, V, and rows of queries where there are any).
// For the kernel, its launch, and a check on the host.
#pragma once

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>

namespace jfkv {
namespace kv8 {
namespace append {

// A table of angles that outgrows an XCD's L2 (4 MB) is read by all heads and parts of a
// block of tokens one after the other on one XCD: 65,535 rows, 34 MB of angles, 327 -> 318
// us, 848 MB read for 1,133.  (Few blocks would be shared out unevenly: 2,048 rows, 0.5 MB,
// take 15.4 us in the grid's order, 15.0 to 16.9 with a block's heads on one XCD.)
constexpr uint32_t kXcds = 8;
constexpr int64_t kTableTogether = 4 << 20;

// Blocks of `block` tokens that total_tok rows of B requests can touch: one per row at
// most, and whole blocks plus two partial ones per request.
inline int64_t units_of(int32_t total, int32_t B, int32_t block) {
  return std::min<int64_t>(total, total / block + 2 * (int64_t)B);
}
// The launch's units, and whether a unit's heads and parts lie together on an XCD.
struct Grid {
  int64_t units;
  bool together;
};
inline Grid grid_of(int32_t total, int32_t B, int32_t block, int32_t rot_dim, int32_t heads, int32_t parts) {
  const int64_t units = units_of(total, B, block), whole = (units + kXcds - 1) / kXcds * kXcds;
  // (place_of counts blocks in 32 bits)
  const bool together =
      (int64_t)total * rot_dim * 4 > kTableTogether && whole * heads * parts <= (int64_t)1 << 32;
  return {together ? whole : units, together};
}

// What the grid's block (x, y, z) takes where they do: blocks are started in the order of
// `at`, on one XCD after the other.
struct Place {
  int unit, head, part;
};
__host__ __device__ __forceinline__ Place place_of(uint32_t x, uint32_t y, uint32_t z, uint32_t units,
                                                   uint32_t heads, uint32_t parts) {
  const uint32_t at = x + units * (y + heads * z), slot = at / kXcds, each = heads * parts;
  return {(int)(slot / each * kXcds + at % kXcds), (int)(slot % each % heads), (int)(slot % each / heads)};
}

// The tokens whose queries block (unit, h) takes: together, a unit takes a run of tokens
// and block h of its `heads` every `heads`-th of them; else all blocks take turns.
struct Tokens {
  int64_t first, end, step;
};
__host__ __device__ __forceinline__ Tokens tokens_of(bool together, int unit, int units, int h, int heads,
                                                     int total) {
  const int64_t run = (total + (int64_t)units - 1) / units, to = (unit + 1) * run;
  return {together ? unit * run + h : h * (int64_t)units + unit,
          together && to < total ? to : (int64_t)total, together ? heads : (int64_t)heads * units};
}

}  // namespace append
}  // namespace kv8
}  // namespace jfkv
