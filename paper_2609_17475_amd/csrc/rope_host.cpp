// C entry points of the rotary positions: argument validation, the frequencies, and
// dispatch.  A call that fails validation launches nothing.
#include <algorithm>
#include <cmath>
#include <cstdint>

#include "jfkv_internal.h"
#include "jfkv_kv8_checks.h"

namespace {

using jfkv::device_status;
using jfkv::fail;
using jfkv::ok;
using jfkv::RopeRows;
using namespace jfkv::kv8;

constexpr int32_t kMaxDim = 65536;

jf_status check_rot(int32_t rot_dim) {
  if (rot_dim < 2 || rot_dim % 2) return fail(JF_ERR_INVALID, "rot_dim %d must be even and positive", rot_dim);
  if (rot_dim > kMaxDim) return fail(JF_ERR_UNSUPPORTED, "rot_dim %d above %d", rot_dim, kMaxDim);
  return JF_OK;
}

jf_status check_rope(const jf_rope* r, int32_t head_dim, int32_t total_tok) {
  if (!r) return fail(JF_ERR_INVALID, "rope is NULL");
  jf_status st = check_rot(r->rot_dim);
  if (st) return st;
  if (r->order != JF_ROPE_HALVES && r->order != JF_ROPE_PAIRS)
    return fail(JF_ERR_UNSUPPORTED, "order %d is neither JF_ROPE_HALVES nor JF_ROPE_PAIRS", r->order);
  if (r->rot_dim > head_dim)
    return fail(JF_ERR_INVALID, "rot_dim %d exceeds head_dim %d", r->rot_dim, head_dim);
  if (total_tok < 0) return fail(JF_ERR_INVALID, "total_tok must be >= 0");
  if (total_tok == 0) return JF_OK;
  if (!r->table || r->table_rows <= 0) return fail(JF_ERR_INVALID, "the table is NULL or has no rows");
  if (misaligned(r->table, 8) || misaligned(r->rows, 4))
    return fail(JF_ERR_INVALID, "the table must be 8-byte aligned, rows 4-byte");
  if (!r->rows && r->table_rows < total_tok)
    return fail(JF_ERR_INVALID, "table_rows %d below total_tok %d, and rows is NULL", r->table_rows, total_tok);
  return JF_OK;
}

jf_status check_stride(int64_t stride, int64_t least, int32_t total_tok, const char* name) {
  // (a token's elements are counted in 64 bits)
  if (stride < 0 || (total_tok > 1 && stride < least) || stride > (int64_t)1 << 31)
    return fail(JF_ERR_INVALID, "%s must be at least heads * head_dim and at most 2^31", name);
  return JF_OK;
}

jf_status check_rows(const RopeRows& x, int32_t head_dim, int32_t total_tok, const char* name) {
  if (x.heads < 0) return fail(JF_ERR_INVALID, "negative number of heads");
  if (x.heads == 0 || total_tok == 0) return JF_OK;
  if ((int64_t)x.heads * head_dim > (int64_t)1 << 24)
    return fail(JF_ERR_UNSUPPORTED, "heads * head_dim above 2^24");
  if (!x.from || !x.to) return fail(JF_ERR_INVALID, "%s or its output is NULL", name);
  if (misaligned(x.from, 2) || misaligned(x.to, 2))
    return fail(JF_ERR_INVALID, "%s and its output must be aligned to an element", name);
  jf_status st;
  if ((st = check_stride(x.from_stride, (int64_t)x.heads * head_dim, total_tok, "a stride")) ||
      (st = check_stride(x.to_stride, (int64_t)x.heads * head_dim, total_tok, "a stride")))
    return st;
  if (x.from == x.to && total_tok > 1 && x.from_stride != x.to_stride)
    return fail(JF_ERR_INVALID, "%s in place needs one stride", name);
  return JF_OK;
}

}  // namespace

jf_status jf_rope_frequencies(int32_t rot_dim, double base, int32_t scaling, double factor,
                              int32_t original_len, double fast, double slow, float* inv_freq,
                              float* magnitude) {
  jf_status st = check_rot(rot_dim);
  if (st) return st;
  if (scaling < JF_ROPE_PLAIN || scaling > JF_ROPE_PARTS)
    return fail(JF_ERR_UNSUPPORTED, "unknown scaling %d", scaling);
  if (!inv_freq || !magnitude) return fail(JF_ERR_INVALID, "NULL output pointer");
  if (!(base > 1.0) || !std::isfinite(base)) return fail(JF_ERR_INVALID, "base must be finite and above 1");
  if (scaling != JF_ROPE_PLAIN && (!(factor > 0.0) || !std::isfinite(factor)))
    return fail(JF_ERR_INVALID, "factor must be finite and positive");
  if (scaling == JF_ROPE_BASE && rot_dim < 4)
    return fail(JF_ERR_INVALID, "a changed base needs a rot_dim of 4 at least");
  double lo = 0.0, hi = 0.0;
  if (scaling == JF_ROPE_PARTS) {
    if (original_len < 1 || !(slow > 0.0) || !(fast > slow) || !std::isfinite(fast))
      return fail(JF_ERR_INVALID, "original_len must be positive, and fast > slow > 0");
    const auto pair_of = [&](double turns) {
      return rot_dim * std::log(original_len / (turns * 2.0 * M_PI)) / (2.0 * std::log(base));
    };
    lo = std::max(std::floor(pair_of(fast)), 0.0);
    hi = std::min(std::ceil(pair_of(slow)), rot_dim - 1.0);
  }
  const double b = scaling == JF_ROPE_BASE ? base * std::pow(factor, rot_dim / (rot_dim - 2.0)) : base;
  *magnitude = scaling == JF_ROPE_PARTS && factor > 1.0 ? (float)(0.1 * std::log(factor) + 1.0) : 1.0f;
  for (int32_t i = 0; i < rot_dim / 2; ++i) {
    const double f = std::pow(b, -2.0 * i / rot_dim);
    double slowed = 0.0;  // the share that is divided by factor
    if (scaling == JF_ROPE_LINEAR) slowed = 1.0;
    if (scaling == JF_ROPE_PARTS)
      // (no ramp where all pairs lie on one side of it: behind its end, they are divided)
      slowed = hi > lo ? std::min(std::max((i - lo) / (hi - lo), 0.0), 1.0) : (i >= hi ? 1.0 : 0.0);
    inv_freq[i] = (float)(slowed > 0.0 ? f * (1.0 - slowed) + f / factor * slowed : f);
  }
  return ok();
}

jf_status jf_rope_table(const int32_t* positions, int32_t n, const float* inv_freq, int32_t rot_dim,
                        float magnitude, float* table, hipStream_t stream) {
  jf_status st = check_rot(rot_dim);
  if (st) return st;
  if (n < 0) return fail(JF_ERR_INVALID, "n must be >= 0");
  if (!std::isfinite(magnitude)) return fail(JF_ERR_INVALID, "magnitude must be finite");
  if (n == 0) return ok();
  if (!positions || !inv_freq || !table) return fail(JF_ERR_INVALID, "NULL device pointer");
  if (misaligned(positions, 4) || misaligned(inv_freq, 4) || misaligned(table, 8))
    return fail(JF_ERR_INVALID, "the table must be 8-byte aligned, positions and inv_freq 4-byte");
  if ((int64_t)n * (rot_dim / 2) + 255 > kMaxThreads)
    return fail(JF_ERR_UNSUPPORTED, "n * rot_dim too large for one launch");
  return device_status(jfkv::launch_rope_table(positions, n, inv_freq, rot_dim, magnitude, table, stream),
                       "rope table launch");
}

jf_status jf_rope_rotate(const jf_rope* rope, int32_t dtype, int32_t head_dim, int32_t transpose,
                         const void* q, int64_t q_stride, void* q_out, int64_t q_out_stride,
                         int32_t num_q_heads, const void* k, int64_t k_stride, void* k_out,
                         int64_t k_out_stride, int32_t num_k_heads, int32_t total_tok,
                         hipStream_t stream) {
  jf_status st = check_dtype(dtype);
  if (st) return st;
  if (head_dim <= 0 || head_dim % 2)
    return fail(JF_ERR_INVALID, "head_dim %d must be even and positive", head_dim);
  if (head_dim > kMaxDim) return fail(JF_ERR_UNSUPPORTED, "head_dim %d above %d", head_dim, kMaxDim);
  const RopeRows a{q, q_out, q_stride, q_out_stride, num_q_heads};
  const RopeRows b{k, k_out, k_stride, k_out_stride, num_k_heads};
  if ((st = check_rope(rope, head_dim, total_tok)) || (st = check_rows(a, head_dim, total_tok, "q")) ||
      (st = check_rows(b, head_dim, total_tok, "k")))
    return st;
  if (total_tok == 0 || num_q_heads + num_k_heads == 0) return ok();
  if ((int64_t)std::max(total_tok, 4096) * 64 + 255 > kMaxThreads)
    return fail(JF_ERR_UNSUPPORTED, "total_tok %d too large for one launch", total_tok);
  return device_status(jfkv::launch_rope_rotate(*rope, dtype == JF_BF16, transpose != 0, head_dim,
                                                num_q_heads ? a : RopeRows{}, num_k_heads ? b : RopeRows{},
                                                total_tok, stream),
                       "rope rotate launch");
}

jf_status jf_kv8_rope_append(const jf_kv_layout* layout, const jf_kv_pool_ptrs* pool, int32_t dtype,
                             const jf_rope* rope, const void* k_new, int64_t k_stride,
                             const void* v_new, int64_t v_stride, const void* q, int64_t q_stride,
                             void* q_out, int32_t num_q_heads, const int32_t* cu_tok,
                             const int32_t* start_pos, const int32_t* block_tables, int32_t B,
                             int32_t max_pages, int32_t total_tok, hipStream_t stream) {
  jf_status st = check_layout(layout);
  if (st) return st;
  if ((st = check_pool(pool)) || (st = check_dtype(dtype)) || (st = check_tables(layout, B, max_pages)) ||
      (st = check_rope(rope, layout->head_dim, total_tok)))
    return st;
  if (rope->rot_dim % 16)
    return fail(JF_ERR_UNSUPPORTED, "rot_dim %d is not a multiple of 16 (rotate, then append)", rope->rot_dim);
  if (total_tok == 0) return ok();
  if (!k_new || !v_new || !cu_tok || !start_pos || !block_tables)
    return fail(JF_ERR_INVALID, "NULL device pointer");
  if (!q != !q_out) return fail(JF_ERR_INVALID, "q and q_out are given both or neither");
  if (misaligned(k_new, 16) || misaligned(v_new, 16) || misaligned(q, 16) || misaligned(q_out, 16))
    return fail(JF_ERR_INVALID, "k_new, v_new, q and q_out must be 16-byte aligned");
  const int64_t kv_row = (int64_t)layout->num_kv_heads * layout->head_dim;
  if ((st = check_stride(k_stride, kv_row, total_tok, "k_stride")) ||
      (st = check_stride(v_stride, kv_row, total_tok, "v_stride")))
    return st;
  if (k_stride % 8 || v_stride % 8)
    return fail(JF_ERR_INVALID, "k_stride and v_stride must be multiples of 8 elements");
  if (q) {
    if ((st = check_heads(layout, num_q_heads))) return st;
    const int64_t q_row = (int64_t)num_q_heads * layout->head_dim;
    if (q_row > (int64_t)1 << 24) return fail(JF_ERR_UNSUPPORTED, "num_q_heads * head_dim above 2^24");
    if ((st = check_stride(q_stride, q_row, total_tok, "q_stride"))) return st;
    if (q_stride % 8) return fail(JF_ERR_INVALID, "q_stride must be a multiple of 8 elements");
    if (q == q_out && total_tok > 1 && q_stride != q_row)
      return fail(JF_ERR_INVALID, "q in place must have no gaps");
  }
  if (((int64_t)total_tok / layout->group_size + 2 * (int64_t)B + 7) * 256 > kMaxThreads)
    return fail(JF_ERR_UNSUPPORTED, "total_tok %d too large for one launch", total_tok);
  return device_status(jfkv::launch_kv8_rope_append(*layout, *pool, dtype == JF_BF16, *rope, k_new,
                                                    k_stride, v_new, v_stride, q, q_stride, q_out,
                                                    q ? num_q_heads : 0, cu_tok, start_pos,
                                                    block_tables, B, max_pages, total_tok, stream),
                       "kv8 rope append launch");
}
