// C entry points of the 8-bit cache: argument validation and dispatch.  A call
// that fails validation launches nothing.
#include <algorithm>
#include <climits>
#include <cmath>
#include <cstdint>

#include "jfkv_internal.h"

namespace {

using jfkv::device_status;
using jfkv::fail;
using jfkv::ok;

// HIP counts the threads of a launch in 32 bits along x.
constexpr int64_t kMaxThreads = ((int64_t)1 << 32) - 1;
constexpr int32_t kMaxGridYZ = 65535;

jf_status check_layout(const jf_kv_layout* L) {
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

jf_status check_pool(const jf_kv_pool_ptrs* p) {
  if (!p || !p->k_codes || !p->k_meta || !p->v_codes || !p->v_meta)
    return fail(JF_ERR_INVALID, "pool pointers must be non-NULL");
  if (((uintptr_t)p->k_codes | (uintptr_t)p->v_codes) & 15)
    return fail(JF_ERR_INVALID, "pool codes must be 16-byte aligned");
  return JF_OK;
}

jf_status check_dtype(int32_t dtype) {
  if (dtype != JF_F16 && dtype != JF_BF16)
    return fail(JF_ERR_UNSUPPORTED, "dtype %d is neither JF_F16 nor JF_BF16", dtype);
  return JF_OK;
}

bool misaligned(const void* p, uintptr_t to) { return ((uintptr_t)p & (to - 1)) != 0; }

jf_status check_scale(float s) {
  // (times log2 e it has to stay finite)
  if (!(std::fabs(s) < 0x1p126f))
    return fail(JF_ERR_INVALID, "softmax_scale must be finite and below 2^126 in magnitude");
  return JF_OK;
}

jf_status check_heads(const jf_kv_layout* L, int32_t num_q_heads) {
  if (num_q_heads <= 0 || num_q_heads % L->num_kv_heads)
    return fail(JF_ERR_INVALID, "num_q_heads %d is not a positive multiple of num_kv_heads %d",
                num_q_heads, L->num_kv_heads);
  return JF_OK;
}

// Tables of B requests, whose positions are counted in 32 bits (with room for
// the last tile).
jf_status check_tables(const jf_kv_layout* L, int32_t B, int32_t max_pages) {
  if (B <= 0 || max_pages <= 0) return fail(JF_ERR_INVALID, "B and max_pages must be positive");
  if ((int64_t)max_pages * L->page_size > INT32_MAX - 16384)
    return fail(JF_ERR_INVALID, "max_pages * page_size overflows int32");
  return JF_OK;
}

// Sizes of a chunk: T rows after prefix_len positions.
jf_status check_chunk(const jf_kv_layout* L, int32_t T, int32_t num_q_heads, int32_t prefix_len) {
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

jf_status check_chunk_table(const jf_kv_layout* L, int32_t T, int32_t prefix_len, int32_t max_pages) {
  if ((int64_t)prefix_len + T > (int64_t)max_pages * L->page_size)
    return fail(JF_ERR_INVALID, "prefix_len %d + T %d exceed max_pages %d * page_size %d", prefix_len,
                T, max_pages, L->page_size);
  return JF_OK;
}

}  // namespace

jf_status jf_kv8_pool_bytes(const jf_kv_layout* layout, size_t* codes_bytes, size_t* exps_bytes) {
  jf_status st = check_layout(layout);
  if (st) return st;
  if (!codes_bytes || !exps_bytes) return fail(JF_ERR_INVALID, "NULL output pointer");
  const size_t slots = (size_t)layout->num_pages * layout->num_kv_heads * layout->page_size;
  *codes_bytes = slots * layout->head_dim;
  *exps_bytes = slots / layout->group_size;
  return ok();
}

jf_status jf_kv8_append(const jf_kv_layout* layout, const jf_kv_pool_ptrs* pool, int32_t dtype,
                        const void* k_new, const void* v_new, const int32_t* cu_tok,
                        const int32_t* start_pos, const int32_t* block_tables, int32_t B,
                        int32_t max_pages, int32_t total_tok, hipStream_t stream) {
  jf_status st = check_layout(layout);
  if (st) return st;
  if ((st = check_pool(pool)) || (st = check_dtype(dtype)) || (st = check_tables(layout, B, max_pages)))
    return st;
  if (total_tok < 0) return fail(JF_ERR_INVALID, "total_tok must be >= 0");
  if (total_tok == 0) return ok();
  if (!k_new || !v_new || !cu_tok || !start_pos || !block_tables)
    return fail(JF_ERR_INVALID, "NULL device pointer");
  if (misaligned(k_new, 16) || misaligned(v_new, 16))
    return fail(JF_ERR_INVALID, "k_new and v_new must be 16-byte aligned");
  if (((int64_t)total_tok / layout->group_size + 2 * (int64_t)B) * 256 > kMaxThreads)
    return fail(JF_ERR_UNSUPPORTED, "total_tok %d too large for one launch", total_tok);
  return device_status(jfkv::launch_kv8_append(*layout, *pool, dtype == JF_BF16, k_new, v_new, cu_tok,
                                               start_pos, block_tables, B, max_pages, total_tok, stream),
                       "kv8 append launch");
}

jf_status jf_kv8_decode_workspace_bytes(const jf_kv_layout* layout, int32_t B, int32_t num_queries,
                                        int32_t num_q_heads, int32_t max_splits,
                                        int32_t weight_pages, size_t* bytes) {
  jf_status st = check_layout(layout);
  if (st) return st;
  if (!bytes) return fail(JF_ERR_INVALID, "NULL output pointer");
  if (B <= 0 || weight_pages < 0) return fail(JF_ERR_INVALID, "B must be positive, weight_pages >= 0");
  if ((int64_t)weight_pages * layout->page_size > INT32_MAX - 16384)
    return fail(JF_ERR_INVALID, "weight_pages * page_size overflows int32");
  if ((st = check_heads(layout, num_q_heads))) return st;
  if (num_queries < 1 || num_queries > 4)
    return fail(JF_ERR_UNSUPPORTED, "num_queries %d outside 1..4", num_queries);
  if (max_splits <= 0 || max_splits > 1024) return fail(JF_ERR_INVALID, "max_splits must be 1..1024");
  if (B > kMaxGridYZ || (int64_t)B * num_q_heads * num_queries > jfkv::kDecodeMaxHeads)
    return fail(JF_ERR_UNSUPPORTED, "B above %d or B * num_q_heads * num_queries above %d", kMaxGridYZ,
                jfkv::kDecodeMaxHeads);
  *bytes = jfkv::kv8_workspace(B, num_queries, num_q_heads, layout->head_dim, max_splits,
                               (int64_t)weight_pages * layout->page_size)
               .bytes;
  return ok();
}

jf_status jf_kv8_decode_attn(const jf_kv_layout* layout, const jf_kv_pool_ptrs* pool, int32_t dtype,
                             const void* q, int32_t B, int32_t num_queries, int32_t num_q_heads,
                             const int32_t* block_tables, int32_t max_pages,
                             const int32_t* seq_lens, float softmax_scale, int32_t max_splits,
                             void* workspace, size_t workspace_bytes, void* out, float* weights,
                             int64_t weights_stride, hipStream_t stream) {
  jf_status st = check_layout(layout);
  if (st) return st;
  if ((st = check_pool(pool)) || (st = check_dtype(dtype)) ||
      (st = check_tables(layout, B, max_pages)) || (st = check_scale(softmax_scale)))
    return st;
  size_t need = 0;
  if ((st = jf_kv8_decode_workspace_bytes(layout, B, num_queries, num_q_heads, max_splits,
                                          weights ? max_pages : 0, &need)))
    return st;
  if (!q || !block_tables || !seq_lens || !workspace || !out)
    return fail(JF_ERR_INVALID, "NULL device pointer");
  if (misaligned(q, 16) || misaligned(out, 16) || misaligned(workspace, 16) || misaligned(weights, 4))
    return fail(JF_ERR_INVALID, "q, out and workspace must be 16-byte aligned, weights 4-byte");
  if (workspace_bytes < need)
    return fail(JF_ERR_INVALID, "workspace %zu bytes < required %zu", workspace_bytes, need);
  if (weights && weights_stride < (int64_t)max_pages * layout->page_size)
    return fail(JF_ERR_INVALID, "weights_stride below max_pages * page_size");
  return device_status(jfkv::launch_kv8_decode(*layout, *pool, dtype == JF_BF16, q, B, num_queries,
                                               num_q_heads, block_tables, max_pages, seq_lens,
                                               softmax_scale, max_splits, workspace, out, weights,
                                               weights_stride, stream),
                       "kv8 decode launch");
}

jf_status jf_kv8_prefill_workspace_bytes(const jf_kv_layout* layout, int32_t T, int32_t num_q_heads,
                                         int32_t prefix_len, size_t* bytes) {
  jf_status st = check_layout(layout);
  if (st) return st;
  if ((st = check_chunk(layout, T, num_q_heads, prefix_len))) return st;
  if (!bytes) return fail(JF_ERR_INVALID, "NULL output pointer");
  *bytes = 0;
  if (T)
    *bytes = jfkv::kv8_prefill_bytes(*layout, T, num_q_heads,
                                     jfkv::kv8_prefill_splits(*layout, T, num_q_heads, prefix_len));
  return ok();
}

jf_status jf_kv8_prefill_attn(const jf_kv_layout* layout, const jf_kv_pool_ptrs* pool, int32_t dtype,
                              const void* q, int32_t T, int32_t num_q_heads,
                              const int32_t* block_table, int32_t max_pages, int32_t prefix_len,
                              float softmax_scale, void* workspace, size_t workspace_bytes, void* out,
                              float* lse, hipStream_t stream) {
  jf_status st = check_layout(layout);
  if (st) return st;
  if ((st = check_pool(pool)) || (st = check_dtype(dtype)) ||
      (st = check_tables(layout, 1, max_pages)) ||
      (st = check_chunk(layout, T, num_q_heads, prefix_len)) ||
      (st = check_chunk_table(layout, T, prefix_len, max_pages)) || (st = check_scale(softmax_scale)))
    return st;
  if (T == 0) return ok();
  if (!q || !block_table || !out) return fail(JF_ERR_INVALID, "NULL device pointer");
  if (misaligned(q, 16) || misaligned(out, 16) || misaligned(lse, 4))
    return fail(JF_ERR_INVALID, "q and out must be 16-byte aligned, lse 4-byte");
  int splits = 1;
  if (workspace) {
    splits = jfkv::kv8_prefill_splits(*layout, T, num_q_heads, prefix_len);
    const size_t need = jfkv::kv8_prefill_bytes(*layout, T, num_q_heads, splits);
    if (workspace_bytes < need)
      return fail(JF_ERR_INVALID, "workspace %zu bytes < required %zu", workspace_bytes, need);
    if (misaligned(workspace, 16)) return fail(JF_ERR_INVALID, "workspace must be 16-byte aligned");
  }
  return device_status(jfkv::launch_kv8_prefill(*layout, *pool, dtype == JF_BF16, q, T, num_q_heads,
                                                block_table, prefix_len, softmax_scale, splits,
                                                workspace, out, lse, stream),
                       "kv8 prefill launch");
}

jf_status jf_kv8_attn_weights(const jf_kv_layout* layout, const jf_kv_pool_ptrs* pool, int32_t dtype,
                              const void* q, const float* lse, int32_t T, int32_t num_q_heads,
                              const int32_t* block_table, int32_t max_pages, int32_t prefix_len,
                              float softmax_scale, float* weights, int64_t weights_stride,
                              hipStream_t stream) {
  jf_status st = check_layout(layout);
  if (st) return st;
  if ((st = check_pool(pool)) || (st = check_dtype(dtype)) ||
      (st = check_tables(layout, 1, max_pages)) ||
      (st = check_chunk(layout, T, num_q_heads, prefix_len)) ||
      (st = check_chunk_table(layout, T, prefix_len, max_pages)) || (st = check_scale(softmax_scale)))
    return st;
  if (T == 0) return ok();
  if (!q || !lse || !block_table || !weights) return fail(JF_ERR_INVALID, "NULL device pointer");
  if (misaligned(q, 16) || misaligned(lse, 4) || misaligned(weights, 4))
    return fail(JF_ERR_INVALID, "q must be 16-byte aligned, lse and weights 4-byte");
  if (weights_stride < (int64_t)prefix_len + T)
    return fail(JF_ERR_INVALID, "weights_stride below prefix_len + T");
  return device_status(jfkv::launch_kv8_weights(*layout, *pool, dtype == JF_BF16, q, lse, T,
                                                num_q_heads, block_table, prefix_len, softmax_scale,
                                                weights, weights_stride, stream),
                       "kv8 weights launch");
}

jf_status jf_kv8_evict_workspace_bytes(const jf_kv_layout* layout, int32_t B, int32_t max_pages,
                                       int32_t keep, size_t* bytes) {
  jf_status st = check_layout(layout);
  if (st) return st;
  if ((st = check_tables(layout, B, max_pages))) return st;
  if (keep <= 0) return fail(JF_ERR_INVALID, "keep must be positive");
  if (!bytes) return fail(JF_ERR_INVALID, "NULL output pointer");
  if (B > kMaxGridYZ) return fail(JF_ERR_UNSUPPORTED, "B above %d", kMaxGridYZ);
  *bytes = jfkv::kv8_evict_bytes(*layout, B, max_pages);
  return ok();
}

jf_status jf_kv8_evict(const jf_kv_layout* layout, const jf_kv_pool_ptrs* pool, int32_t B,
                       const int32_t* block_tables, int32_t max_pages, const int32_t* seq_lens,
                       const float* weights, int64_t weights_stride, int32_t keep, int32_t recent,
                       const int32_t* dst_tables, int32_t dst_max_pages, void* workspace,
                       size_t workspace_bytes, int32_t* kept, float* kept_weights,
                       hipStream_t stream) {
  jf_status st = check_layout(layout);
  if (st) return st;
  size_t need = 0;
  if ((st = check_pool(pool)) ||
      (st = jf_kv8_evict_workspace_bytes(layout, B, max_pages, keep, &need)))
    return st;
  if (recent < 0 || recent > keep) return fail(JF_ERR_INVALID, "recent must be 0 .. keep");
  if (dst_max_pages <= 0 || (int64_t)dst_max_pages * layout->page_size < keep)
    return fail(JF_ERR_INVALID, "keep %d exceeds dst_max_pages %d * page_size %d", keep, dst_max_pages,
                layout->page_size);
  if ((int64_t)B * layout->num_kv_heads * 256 > kMaxThreads)
    return fail(JF_ERR_UNSUPPORTED, "B * num_kv_heads too large for one launch");
  // blocks of the positions that can stay, K's and V's, of 256 threads at most;
  // and room for the strides of loops that count to keep in 32 bits
  const int64_t most = std::min<int64_t>(keep, (int64_t)max_pages * layout->page_size);
  if (keep > INT32_MAX / 2 || (most / layout->group_size + 1) * 2 * 256 > kMaxThreads)
    return fail(JF_ERR_UNSUPPORTED, "keep %d too large for one launch", keep);
  if (!block_tables || !seq_lens || !weights || !dst_tables || !kept || !kept_weights ||
      (need && !workspace))
    return fail(JF_ERR_INVALID, "NULL device pointer");
  if (misaligned(workspace, 16) || misaligned(weights, 4) || misaligned(kept, 4) || misaligned(kept_weights, 4))
    return fail(JF_ERR_INVALID, "workspace must be 16-byte aligned, weights and outputs 4-byte");
  if (workspace_bytes < need)
    return fail(JF_ERR_INVALID, "workspace %zu bytes < required %zu", workspace_bytes, need);
  if (weights_stride < (int64_t)max_pages * layout->page_size)
    return fail(JF_ERR_INVALID, "weights_stride below max_pages * page_size");
  return device_status(jfkv::launch_kv8_evict(*layout, *pool, B, block_tables, max_pages, seq_lens,
                                              weights, weights_stride, keep, recent, dst_tables,
                                              dst_max_pages, workspace, kept, kept_weights,
                                              stream),
                       "kv8 evict launch");
}
