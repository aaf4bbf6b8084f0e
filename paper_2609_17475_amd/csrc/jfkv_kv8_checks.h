// Checks of arguments that the entry points of the 8-bit cache and of the operators
// around it share.  Each reports what it refuses and returns its status.
#pragma once

#include <climits>
#include <cmath>
#include <cstdint>

#include "jfkv_internal.h"

namespace jfkv {
namespace kv8 {

// HIP counts the threads of a launch in 32 bits along x.
constexpr int64_t kMaxThreads = ((int64_t)1 << 32) - 1;
constexpr int32_t kMaxGridYZ = 65535;

inline jf_status check_layout(const jf_kv_layout* L) {
  if (!L) return fail(JF_ERR_INVALID, "layout is NULL");
  if (L->page_size <= 0 || L->num_kv_heads <= 0 || L->head_dim <= 0 || L->group_size <= 0 ||
      L->num_pages <= 0)
    return fail(JF_ERR_INVALID, "layout fields must be positive");
  const bool d_ok = L->head_dim == 64 || L->head_dim == 128 || L->head_dim == 256;
  const bool g_ok = L->group_size == 16 || L->group_size == 32 || L->group_size == 64 ||
                    L->group_size == 128;
  if (!d_ok || !g_ok || L->page_size % 64 || L->page_size > 4096 || L->page_size % L->group_size)
    return fail(JF_ERR_UNSUPPORTED,
                "unsupported geometry (page_size %d must be a multiple of 64 and <= 4096, head_dim "
                "%d in {64,128,256}, group_size %d (positions per exponent) in {16,32,64,128} and a "
                "divisor of page_size)",
                L->page_size, L->head_dim, L->group_size);
  if (L->num_kv_heads > kMaxGridYZ || (int64_t)L->num_pages * L->num_kv_heads > INT32_MAX)
    return fail(JF_ERR_UNSUPPORTED, "num_kv_heads above %d or num_pages * num_kv_heads above 2^31 - 1",
                kMaxGridYZ);
  return JF_OK;
}

inline jf_status check_pool(const jf_kv_pool_ptrs* p) {
  if (!p || !p->k_codes || !p->k_meta || !p->v_codes || !p->v_meta)
    return fail(JF_ERR_INVALID, "pool pointers must be non-NULL");
  if (((uintptr_t)p->k_codes | (uintptr_t)p->v_codes) & 15)
    return fail(JF_ERR_INVALID, "pool codes must be 16-byte aligned");
  return JF_OK;
}

inline jf_status check_dtype(int32_t dtype) {
  if (dtype != JF_F16 && dtype != JF_BF16)
    return fail(JF_ERR_UNSUPPORTED, "dtype %d is neither JF_F16 nor JF_BF16", dtype);
  return JF_OK;
}

inline bool misaligned(const void* p, uintptr_t to) { return ((uintptr_t)p & (to - 1)) != 0; }

inline jf_status check_scale(float s) {
  // (times log2 e it has to stay finite)
  if (!(std::fabs(s) < 0x1p126f))
    return fail(JF_ERR_INVALID, "softmax_scale must be finite and below 2^126 in magnitude");
  return JF_OK;
}

inline jf_status check_heads(const jf_kv_layout* L, int32_t num_q_heads) {
  if (num_q_heads <= 0 || num_q_heads % L->num_kv_heads)
    return fail(JF_ERR_INVALID, "num_q_heads %d is not a positive multiple of num_kv_heads %d",
                num_q_heads, L->num_kv_heads);
  return JF_OK;
}

// Tables of B requests, whose positions are counted in 32 bits (with room for
// the last tile).
inline jf_status check_tables(const jf_kv_layout* L, int32_t B, int32_t max_pages) {
  if (B <= 0 || max_pages <= 0) return fail(JF_ERR_INVALID, "B and max_pages must be positive");
  if ((int64_t)max_pages * L->page_size > INT32_MAX - 16384)
    return fail(JF_ERR_INVALID, "max_pages * page_size overflows int32");
  return JF_OK;
}

// Sizes of a chunk: T rows after prefix_len positions.
inline jf_status check_chunk(const jf_kv_layout* L, int32_t T, int32_t num_q_heads, int32_t prefix_len) {
  if (T < 0 || prefix_len < 0) return fail(JF_ERR_INVALID, "negative size");
  jf_status st = check_heads(L, num_q_heads);
  if (st) return st;
  if ((int64_t)T * num_q_heads > INT32_MAX || (int64_t)T * num_q_heads * (L->head_dim / 4) > kMaxThreads)
    return fail(JF_ERR_UNSUPPORTED, "T * num_q_heads too large for one launch");
  if ((int64_t)prefix_len + T > INT32_MAX - 16384)
    return fail(JF_ERR_INVALID, "prefix_len + T overflows int32");
  if (((int64_t)prefix_len + T + 255) * L->num_kv_heads * 2 > kMaxThreads)
    return fail(JF_ERR_UNSUPPORTED, "the positions of all KV heads are too many for one launch");
  return JF_OK;
}

inline jf_status check_chunk_table(const jf_kv_layout* L, int32_t T, int32_t prefix_len, int32_t max_pages) {
  if ((int64_t)prefix_len + T > (int64_t)max_pages * L->page_size)
    return fail(JF_ERR_INVALID, "prefix_len %d + T %d exceed max_pages %d * page_size %d", prefix_len,
                T, max_pages, L->page_size);
  return JF_OK;
}

}  // namespace kv8
}  // namespace jfkv
