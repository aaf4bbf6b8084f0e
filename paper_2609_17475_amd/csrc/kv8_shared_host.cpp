// C entry points of the attention of requests that share prefixes: argument validation
// and dispatch.  A call that fails validation launches nothing.
#include <cstdint>

#include "jfkv_internal.h"
#include "jfkv_kv8_checks.h"

using jfkv::device_status;
using jfkv::fail;
using jfkv::ok;
using namespace jfkv::kv8;

jf_status jf_kv8_shared_workspace_bytes(const jf_kv_layout* layout, int32_t B, int32_t num_groups,
                                        int32_t num_queries, int32_t num_q_heads, size_t* bytes) {
  jf_status st = check_layout(layout);
  if (st) return st;
  if (!bytes) return fail(JF_ERR_INVALID, "NULL output pointer");
  if (B <= 0 || num_groups <= 0 || num_groups > B)
    return fail(JF_ERR_INVALID, "B must be positive, num_groups 1 .. B");
  if ((st = check_heads(layout, num_q_heads))) return st;
  if (num_queries < 1 || num_queries > 4)
    return fail(JF_ERR_UNSUPPORTED, "num_queries %d outside 1..4", num_queries);
  if (B > kMaxGridYZ || (int64_t)B * num_q_heads * num_queries > jfkv::kDecodeMaxHeads)
    return fail(JF_ERR_UNSUPPORTED, "B above %d or B * num_q_heads * num_queries above %d", kMaxGridYZ,
                jfkv::kDecodeMaxHeads);
  *bytes = jfkv::kv8_shared_bytes(*layout, B, num_groups, num_queries, num_q_heads);
  return ok();
}

jf_status jf_kv8_shared_attn(const jf_kv_layout* layout, const jf_kv_pool_ptrs* pool, int32_t dtype,
                             const void* q, int32_t B, int32_t num_queries, int32_t num_q_heads,
                             const int32_t* block_tables, int32_t max_pages,
                             const int32_t* seq_lens, const int32_t* group_start,
                             const int32_t* shared_lens, int32_t num_groups, float softmax_scale,
                             void* workspace, size_t workspace_bytes, void* out, float* lse,
                             hipStream_t stream) {
  jf_status st = check_layout(layout);
  if (st) return st;
  if ((st = check_pool(pool)) || (st = check_dtype(dtype)) ||
      (st = check_tables(layout, B, max_pages)) || (st = check_scale(softmax_scale)))
    return st;
  size_t need = 0;
  if ((st = jf_kv8_shared_workspace_bytes(layout, B, num_groups, num_queries, num_q_heads, &need)))
    return st;
  if (!q || !block_tables || !seq_lens || !group_start || !shared_lens || !workspace || !out)
    return fail(JF_ERR_INVALID, "NULL device pointer");
  if (misaligned(q, 16) || misaligned(out, 16) || misaligned(workspace, 16) || misaligned(lse, 4))
    return fail(JF_ERR_INVALID, "q, out and workspace must be 16-byte aligned, lse 4-byte");
  if (workspace_bytes < need)
    return fail(JF_ERR_INVALID, "workspace %zu bytes < required %zu", workspace_bytes, need);
  return device_status(jfkv::launch_kv8_shared(*layout, *pool, dtype == JF_BF16, q, B, num_queries,
                                               num_q_heads, block_tables, max_pages, seq_lens,
                                               group_start, shared_lens, num_groups, softmax_scale,
                                               workspace, out, lse, stream),
                       "kv8 shared launch");
}
