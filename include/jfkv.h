/*
 * jfkv.h -- C ABI of libjfkv.so: attention executed directly over a
 * group-wise 4-bit quantized, paged KV cache on AMD Instinct MI355X (gfx950).
 *
 * The operations follow the KVExec component of "JustFit: Just-in-Time State
 * Management for Local LLM Serving":
 *   - a fixed backing pool of 256-token pages, a per-request page table that
 *     maps token order to pages, page IDs returned to a free list on
 *     completion (Background, "Compact histories need reusable storage");
 *   - reference-counted pages shared by requests with a common prefix and
 *     all-or-nothing page reservation (Sec. 3.3, eq. reservation and the
 *     refcounted shared prefixes it describes; Algorithm 1 recycles
 *     zero-reference pages after releasing a request);
 *   - single-query decode that reads the compressed pages directly, and
 *     prefill that consumes the same pages as floating operands (Sec. 3.1,
 *     "Decode and prefill need different kernels"); query heads grouped
 *     over shared KV heads, each head independent (eq. groupattention);
 *   - bounded temporary storage: the decode workspace has a size fixed by
 *     the caller's split cap, independent of context length (Sec. 3.1,
 *     "Finish one head group ..." motivates bounding workspace; eq.
 *     layerbytes is what the fused prefill avoids materializing).
 * Stored format: affine 4-bit codes with one fp16 scale and one fp16 bias
 * per group of head_dim elements (the affine 4-bit format the Introduction
 * describes for weights: a scale and an offset per group), eight codes per 32-bit word
 * (Appendix A, Table codec, per-vector storage).
 *
 * ---------------------------------------------------------------------
 * Pool byte layout (per layer; one set for K and one for V):
 *   k_codes  uint8 [NP][Hkv][P][d/2]          byte j of a position's row =
 *                                             code(2j) | code(2j+1) << 4
 *   v_codes  uint8 [NP][Hkv][P/2][d/4][2][2]  positions paired (2s, 2s+1):
 *                                             dims 4u..4u+3 of slot t are the
 *                                             2 bytes at ((t/2)*(d/4)+u)*4 +
 *                                             (t%2)*2, holding code(4u) |
 *                                             code(4u+1)<<4 and code(4u+2) |
 *                                             code(4u+3)<<4
 *   k_meta, v_meta  fp16 [NP][Hkv][P][d/G][2]  (scale, bias) per group
 * Bytes per position per layer: 2*Hkv*(d/2 + 4*d/G) (1,152 at Hkv=8,
 * d=128, G=64).
 *
 * Quantizer (bit-exact contract), per group x_0..x_{G-1} of fp16 values:
 *   mn, mx   = min, max (binary32; -0 orders below +0)
 *   bias     = fp16 of mn rounded toward -inf
 *   range    = mx - mn; step = range / 15  (binary32, IEEE round-to-nearest)
 *   scale    = fp16 of step rounded toward +inf; +0 when range == 0
 *   code_i   = 0 if scale == 0, else clamp(rint((x_i - bias) / scale), 0, 15)
 *              with the subtraction and division separate binary32 ops and
 *              rint rounding half to even
 *   x^_i     = scale * code_i + bias
 * Inputs must be finite.
 *
 * ---------------------------------------------------------------------
 * Conventions for every entry point:
 *   - Every function returns jf_status; no C++ exception crosses the ABI.
 *   - Arguments are validated before anything is launched; a call that
 *     fails validation has no side effect.  jf_last_error() then returns a
 *     message (thread-local; valid until the next jf_* call on the thread).
 *   - Device pointers are caller-owned (allocated by the caller, e.g. by
 *     PyTorch); the library never allocates or frees device memory.  Device
 *     work is enqueued asynchronously on the given stream (NULL = the
 *     default stream); faults inside kernels surface at the caller's next
 *     synchronization.  A launch failure returns JF_ERR_DEVICE.
 *   - Host page-pool objects are owned by the library from _create until
 *     _destroy and are not thread-safe: callers serialize calls per pool.
 *   - GQA mapping: query head h reads KV head h / (num_q_heads / Hkv).
 */
#ifndef JFKV_H
#define JFKV_H

#include <stddef.h>
#include <stdint.h>

#include <hip/hip_runtime_api.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  JF_OK = 0,
  JF_ERR_INVALID = 1,     /* bad argument (NULL, shape, range)               */
  JF_ERR_NO_PAGES = 2,    /* page reservation could not be satisfied         */
  JF_ERR_DEVICE = 3,      /* HIP launch or runtime error                     */
  JF_ERR_UNSUPPORTED = 4, /* valid but not implemented geometry              */
  JF_ERR_STATE = 5,       /* operation not allowed in the object's state     */
  JF_ERR_IO = 6           /* host file I/O failed (snapshots)                */
} jf_status;

/* Message for the last failing jf_* call on this thread ("" if none). */
const char* jf_last_error(void);

/* Library version string. */
const char* jf_version(void);

/* Pool geometry.  Supported: page_size a multiple of 64 (256 in the paper's
 * geometry); head_dim 64, 128 or 256; group_size 32, 64 or 128 dividing
 * head_dim; num_kv_heads >= 1; num_pages >= 1. */
typedef struct {
  int32_t page_size;
  int32_t num_kv_heads;
  int32_t head_dim;
  int32_t group_size;
  int32_t num_pages;
} jf_kv_layout;

/* Device pointers to one layer's pools (layout above). */
typedef struct {
  void* k_codes;
  void* k_meta;
  void* v_codes;
  void* v_meta;
} jf_kv_pool_ptrs;

/* Bytes of one codes array and of one meta array for the layout (the same
 * for K and V).  Errors: JF_ERR_INVALID / JF_ERR_UNSUPPORTED for bad
 * geometry or NULL outputs. */
jf_status jf_kv_pool_bytes(const jf_kv_layout* layout, size_t* codes_bytes,
                           size_t* meta_bytes);

/* ---------------------------------------------------------------------
 * Host page allocator and per-request page tables (paging: Background,
 * "Compact histories need reusable storage"; shared prefixes and
 * reservation: eq. reservation; recycling: Algorithm 1).
 * ------------------------------------------------------------------- */
typedef struct jf_page_pool jf_page_pool;

/* Create a pool of num_pages page IDs.  The free list is a stack; with
 * shuffle_seed != 0 its initial order is a seeded permutation (so
 * consecutive reservations receive non-contiguous physical pages), with 0
 * pages are handed out in increasing order.  *out receives the pool. */
jf_status jf_page_table_pool_create(int32_t num_pages, int32_t page_size,
                                    uint64_t shuffle_seed, jf_page_pool** out);
jf_status jf_page_table_pool_destroy(jf_page_pool* pool);

/* New empty request (length 0, no pages); *seq receives its handle. */
jf_status jf_page_table_create(jf_page_pool* pool, int32_t* seq);

/* New request that shares (copy-free, reference count + 1) the first
 * prefix_len positions of src.  prefix_len must be a multiple of page_size
 * and at most src's length, so the new request's next write lands on a page
 * of its own.  Its length starts at prefix_len. */
jf_status jf_page_table_fork(jf_page_pool* pool, int32_t src,
                             int32_t prefix_len, int32_t* seq);

/* Append the n given free pages to seq's page list (explicit placement,
 * e.g. a reversed or shuffled mapping).  JF_ERR_STATE if any is not free
 * or listed twice; nothing changes then. */
jf_status jf_page_table_assign(jf_page_pool* pool, int32_t seq,
                               const int32_t* page_ids, int32_t n);

/* Ensure seq owns ceil(new_len / page_size) pages, taking missing ones from
 * the free list; all or nothing (JF_ERR_NO_PAGES leaves seq unchanged).
 * JF_ERR_STATE if positions length..new_len-1 would fall on a page whose
 * reference count is above one (shared pages are read-only). */
jf_status jf_page_table_reserve(jf_page_pool* pool, int32_t seq,
                                int32_t new_len);

/* Commit seq's length after its rows were appended; len must not exceed
 * its page capacity. */
jf_status jf_page_table_set_length(jf_page_pool* pool, int32_t seq,
                                   int32_t len);

/* Drop seq: each of its pages loses one reference; pages reaching zero go
 * back on the free list (last released, first reused).  The handle becomes
 * invalid (JF_ERR_STATE on reuse). */
jf_status jf_page_table_release(jf_page_pool* pool, int32_t seq);

/* Write the page tables of n requests as a host block table
 * [n][max_pages] (unused entries -1) and their lengths [n].  JF_ERR_INVALID
 * if a request has more than max_pages pages. */
jf_status jf_page_table_export(const jf_page_pool* pool, const int32_t* seqs,
                               int32_t n, int32_t max_pages,
                               int32_t* block_table, int32_t* lens);

/* Pages currently free, in use (reference count > 0), and the most pages
 * ever in use at once. */
jf_status jf_page_table_stats(const jf_page_pool* pool, int32_t* free_pages,
                              int32_t* used_pages, int32_t* high_water);

/* Number of pages of seq and its committed length. */
jf_status jf_page_table_info(const jf_page_pool* pool, int32_t seq,
                             int32_t* n_pages, int32_t* length);

/* ---------------------------------------------------------------------
 * Device work.
 * ------------------------------------------------------------------- */

/* Quantize rows of new K and V and write them into their pages (the
 * "pending cache writes" a step finishes before its pages may be released,
 * Algorithm 1).
 *   k_new, v_new  fp16 [total_tok][Hkv][d] (device), rows of all requests
 *                 concatenated;
 *   cu_tok        int32 [B+1] (device) row offsets: request b owns rows
 *                 cu_tok[b] .. cu_tok[b+1]-1, total_tok == cu_tok[B];
 *   start_pos     int32 [B] (device) logical position of each request's
 *                 first new row;
 *   block_tables  int32 [B][max_pages] (device) physical page of each
 *                 logical page.
 * Rows whose logical page is beyond max_pages or whose page ID is outside
 * [0, num_pages) are skipped (nothing is written for them).  The pages must
 * have been reserved and not be shared.  Codes, scales and biases are
 * bit-exact with the quantizer contract above. */
jf_status jf_kv_quantize_append(const jf_kv_layout* layout,
                                const jf_kv_pool_ptrs* pool,
                                const void* k_new, const void* v_new,
                                const int32_t* cu_tok,
                                const int32_t* start_pos,
                                const int32_t* block_tables, int32_t B,
                                int32_t max_pages, int32_t total_tok,
                                hipStream_t stream);

/* Workspace bytes jf_decode_attn_q4 needs: a fixed 262,144-byte region of
 * completion counters (room for B * num_q_heads <= 65,536; larger products
 * return JF_ERR_UNSUPPORTED), then B * num_q_heads * max_splits *
 * (head_dim + 4) * 4 bytes of fp32 partials (o/l, m, l per split, padded to
 * 16-byte records).  It does
 * not depend on sequence lengths. */
jf_status jf_decode_workspace_bytes(int32_t B, int32_t num_q_heads,
                                    int32_t head_dim, int32_t max_splits,
                                    size_t* bytes);

/* Single-query decode attention over the paged 4-bit cache: split-K
 * partials, then a log-sum-exp combine done by the last split of each
 * (request, KV head) to finish; one kernel on `stream`.
 *   q            fp16 [B][num_q_heads][d] (device)
 *   block_tables int32 [B][max_pages] (device)
 *   seq_lens     int32 [B] (device): request b attends to its logical
 *                positions 0..seq_lens[b]-1 (append first, then attend);
 *                values above max_pages*page_size are clamped; a request
 *                with length <= 0 gets an all-zero output row
 *   softmax_scale  logits = softmax_scale * q . k
 *   max_splits   cap on partials per request and KV head (1..1024); a
 *                request with n pages uses S = min(max_splits, n,
 *                max(1, floor(compute units / (num_kv_heads *
 *                ceil(Gq / H))))), H the query heads one block serves:
 *                h = 4 for 32-dim groups or head_dim 256, else 8, and
 *                H = 2h when Gq > h and head_dim <= 128, else h
 *                page-aligned splits of equal page counts, the remainder on
 *                the first (S depends on neither the batch nor the other
 *                requests, so a request's output is the same in any batch)
 *   workspace    device scratch of at least jf_decode_workspace_bytes().
 *                Its first 262,144 bytes (completion counters) must be zero
 *                before the first call, e.g. by allocating it zero-filled;
 *                every call that completes leaves them zero, so the same
 *                workspace serves any later call of any shape that fits.
 *                Calls that may overlap in time must not share one.
 *   out          fp16 [B][num_q_heads][d] (device)
 * Page IDs outside [0, num_pages) are never dereferenced; the positions
 * they would hold do not contribute. */
jf_status jf_decode_attn_q4(const jf_kv_layout* layout,
                            const jf_kv_pool_ptrs* pool, const void* q,
                            int32_t B, int32_t num_q_heads,
                            const int32_t* block_tables, int32_t max_pages,
                            const int32_t* seq_lens, float softmax_scale,
                            int32_t max_splits, void* workspace,
                            size_t workspace_bytes, void* out,
                            hipStream_t stream);

/* Short packed verification (Sec. 3.1, the speculative-verification
 * paragraph after eq. groupattention; Appendix A, "Codec and Attention
 * Dispatch": causal string masks, 2 to 4 queries).  The last num_queries
 * positions of request b (already appended: positions seq_lens[b] -
 * num_queries .. seq_lens[b] - 1) are its query tokens; token k sees the
 * positions 0 .. seq_lens[b] - num_queries + k (a causal mask aligned to the
 * end of the cache).  One page scan serves every token and query head of a
 * KV head chunk, as in jf_decode_attn_q4.
 *   q            fp16 [B][num_queries][num_q_heads][d] (device)
 *   num_queries  1..4 (1 is jf_decode_attn_q4); larger: JF_ERR_UNSUPPORTED
 *   workspace    at least jf_decode_workspace_bytes(B, num_q_heads *
 *                num_queries, d, max_splits); same zeroing rule as decode
 *   out          fp16 [B][num_queries][num_q_heads][d] (device)
 * Other arguments as jf_decode_attn_q4; a token whose visible length is
 * <= 0 gets an all-zero output row. */
jf_status jf_verify_attn_q4(const jf_kv_layout* layout,
                            const jf_kv_pool_ptrs* pool, const void* q,
                            int32_t B, int32_t num_queries, int32_t num_q_heads,
                            const int32_t* block_tables, int32_t max_pages,
                            const int32_t* seq_lens, float softmax_scale,
                            int32_t max_splits, void* workspace,
                            size_t workspace_bytes, void* out,
                            hipStream_t stream);

/* One decode step, append then attend, in one kernel: request b's new row
 * (k_new, v_new: fp16 [B][Hkv][d], device) is quantized into the pool at
 * logical position seq_lens[b] - 1 exactly as jf_kv_quantize_append would
 * write it (same codes, scales, biases and placement; a row whose position
 * is beyond max_pages * page_size or whose page ID is outside
 * [0, num_pages) is not written), and the query then attends to positions
 * 0..seq_lens[b]-1, the new row included, as in jf_decode_attn_q4 (same
 * arguments and workspace).  One launch per decode step instead of two
 * (append, then attend); the outputs and the pool are the same.  The row's
 * page must be reserved and not shared. */
jf_status jf_decode_step_q4(const jf_kv_layout* layout,
                            const jf_kv_pool_ptrs* pool, const void* k_new,
                            const void* v_new, const void* q, int32_t B,
                            int32_t num_q_heads, const int32_t* block_tables,
                            int32_t max_pages, const int32_t* seq_lens,
                            float softmax_scale, int32_t max_splits,
                            void* workspace, size_t workspace_bytes, void* out,
                            hipStream_t stream);

/* jf_decode_step_q4 without a workspace argument, for callers that cannot
 * allocate device memory (code under HIP graph capture, tight serving loops,
 * harnesses that forbid allocation).  The step's completion counters and
 * split records live in a device array inside the library: 8 MiB per device
 * (64 KiB of counters, then records), held until the process ends; its
 * address is looked up once per device (hipGetSymbolAddress, which
 * allocates nothing), and the first call on a device also enqueues a small
 * kernel that zeroes the counters.  The call allocates and frees nothing.
 * Arguments, outputs and pool writes are those of jf_decode_step_q4 with the
 * same max_splits (the outputs are bitwise the same).
 * Limits: B * num_kv_heads * ceil(Gq / 4) <= 16,384 counters and
 * B * num_q_heads * max_splits * (head_dim + 4) * 4 <= 8,323,072 bytes of
 * records; larger requests return JF_ERR_INVALID (nothing launched).
 * Every call on a device shares that device's array and keeps its last
 * contents: calls that may overlap in time on one device (other streams,
 * other threads) race and must not be issued. */
jf_status jf_decode_step_q4_static(const jf_kv_layout* layout,
                                   const jf_kv_pool_ptrs* pool,
                                   const void* k_new, const void* v_new,
                                   const void* q, int32_t B,
                                   int32_t num_q_heads,
                                   const int32_t* block_tables,
                                   int32_t max_pages, const int32_t* seq_lens,
                                   float softmax_scale, int32_t max_splits,
                                   void* out, hipStream_t stream);

/* Chunked-prefill attention for one request: query i of the chunk sits at
 * absolute position prefix_len + i and attends to the dequantized prefix
 * positions 0..prefix_len-1 (through block_table) and, causally, to the
 * chunk's own fp16 rows 0..i.  The chunk is not written to the pool here:
 * call jf_kv_quantize_append afterwards.
 *   q        fp16 [T][num_q_heads][d] (device)
 *   k_chunk, v_chunk  fp16 [T][Hkv][d] (device)
 *   block_table  int32 [max_pages] (device); pages 0..ceil(prefix_len/P)-1
 *                are read; prefix_len must be <= max_pages * page_size
 *   out      fp16 [T][num_q_heads][d] (device)
 * Products run on fp16 matrix cores with fp32 accumulation.  Key codes
 * enter exactly, with scales and biases applied to the fp32 scores; prefix
 * values enter as (scale * code + bias) / 2 split into an fp16 high and low
 * part (exact to ~2^-21 relative, no fp16 overflow for any group), the
 * chunk's own fp16 rows exactly. */
jf_status jf_prefill_attn_q4(const jf_kv_layout* layout,
                             const jf_kv_pool_ptrs* pool, const void* q,
                             const void* k_chunk, const void* v_chunk,
                             int32_t T, int32_t num_q_heads,
                             const int32_t* block_table, int32_t max_pages,
                             int32_t prefix_len, float softmax_scale,
                             void* out, hipStream_t stream);

/* jf_prefill_attn_q4 with device scratch that lets the work be laid evenly
 * over the chip: where the chunk's rows alone would not fill it (a short
 * chunk over a long prefix) or would leave its last turn nearly empty, the
 * keys of a KV head are shared evenly by its blocks, which leave fp32 partial
 * states (o, m, l) in the workspace for a second small kernel to combine.
 * jf_prefill_workspace_bytes gives the bytes such a call needs: 0 where the
 * work is even as it is (the workspace is then not used and may be NULL), and
 * never more than two partial states per compute unit, whatever the lengths
 * (on 256 of them 38 MB at head_dim 64, 71 MB at 128, 69 MB at 256).
 *   workspace  device scratch, 16-byte aligned, of at least that many bytes;
 *              its contents do not matter before the call nor after it.  Calls
 *              that may overlap in time must not share one.
 * Other arguments, outputs and errors as jf_prefill_attn_q4; the outputs are
 * the same up to the order of the fp32 sums. */
jf_status jf_prefill_workspace_bytes(const jf_kv_layout* layout, int32_t T,
                                     int32_t num_q_heads, int32_t prefix_len, size_t* bytes);
jf_status jf_prefill_attn_q4_ws(const jf_kv_layout* layout,
                                const jf_kv_pool_ptrs* pool, const void* q,
                                const void* k_chunk, const void* v_chunk,
                                int32_t T, int32_t num_q_heads,
                                const int32_t* block_table, int32_t max_pages,
                                int32_t prefix_len, float softmax_scale,
                                void* workspace, size_t workspace_bytes,
                                void* out, hipStream_t stream);

/* Page -> operand reconstruction of one head group for an SDPA-style
 * consumer (Background, "Stored format is not execution format", eq.
 * layerbytes; Sec. 3.1, "Finish one head group before starting the next",
 * eq. groupattention): the dequantized K and V vectors of KV heads
 * kv0 .. kv0 + num_heads - 1 at logical positions 0 .. n_pos - 1 of one
 * request, read through block_table, written as contiguous operands.  A
 * grouped prefill reconstructs one group (the paper's: two KV heads),
 * attends with that group's query heads, and reuses the same
 * 2 * num_heads * n_pos * d * 2 bytes for the next group.
 *   block_table  int32 [max_pages] (device); n_pos <= max_pages * page_size
 *   k_out, v_out fp16 [num_heads][n_pos][d] (device, 16-byte aligned,
 *                caller-owned); element = scale * code + bias rounded once to
 *                fp16 (nearest, ties to even: the exact value's rounding,
 *                not a rounding of an fp32 intermediate)
 * A page ID outside [0, num_pages) gives zero vectors.  n_pos = 0 launches
 * nothing. */
jf_status jf_reconstruct_q4(const jf_kv_layout* layout,
                            const jf_kv_pool_ptrs* pool,
                            const int32_t* block_table, int32_t max_pages,
                            int32_t n_pos, int32_t kv0, int32_t num_heads,
                            void* k_out, void* v_out, hipStream_t stream);

/* ------------------------------------------------------- snapshots
 * Prefix snapshots and their restoration (Sec. 3.4, "Keep Checkpointing
 * from Undoing the Savings"; Appendix A, Fig. kv-detail (b); Table writer).
 * A page of one layer's pool is packed as its four runs for all KV heads:
 * K codes, K (scale, bias), V codes, V (scale, bias), exactly as the pool
 * stores them (page_bytes = 2 * Hkv * page_size * (d/2 + 4 * d/G)). */

/* page_bytes of this layout. */
jf_status jf_kv_page_bytes(const jf_kv_layout* layout, size_t* bytes);

/* Pack pages block_table[first .. first+count-1] of one layer's pool, in
 * that order, into buf (count * page_bytes bytes of device memory, 16-byte
 * aligned); or unpack buf into those pages.  block_table: int32 (device).
 * A page ID outside [0, num_pages) packs as zeros and is skipped when
 * unpacking.  One kernel on stream; the pages are read (or written) where
 * they are.  A buf that is not device memory is rejected (JF_ERR_INVALID):
 * kernels never dereference host memory.  Pool codes 16-byte and meta
 * 4-byte aligned. */
jf_status jf_kv_pack_pages(const jf_kv_layout* layout, const jf_kv_pool_ptrs* pool,
                           const int32_t* block_table, int32_t first, int32_t count,
                           void* buf, hipStream_t stream);
jf_status jf_kv_unpack_pages(const jf_kv_layout* layout, const jf_kv_pool_ptrs* pool,
                             const int32_t* block_table, int32_t first, int32_t count,
                             const void* buf, hipStream_t stream);

/* Read-rate calibration (not part of the method): reads bytes (a positive
 * multiple of 16) of device memory at buf once, with the 16-byte
 * non-temporal loads of the HBM-bound kernels, `blocks` blocks of 512
 * threads each reading one contiguous share, and does nothing else.  The
 * time it takes on a buffer of the decode's size is the practical read
 * ceiling the kernels' fractions of peak are compared with.  sink: 4 bytes
 * of device memory (written only for a buffer whose words xor to a fixed
 * 96-bit pattern).  buf 16-byte aligned; blocks 1..65535.  One kernel on
 * stream. */
jf_status jf_calib_read_stream(const void* buf, size_t bytes, int32_t blocks, void* sink,
                               hipStream_t stream);

/* Save the first n_pos positions of one request, all n_layers layers
 * (pools[l]: the layers' pools, one layout), to a file in one pass.  The
 * pages are read in place through block_table (device; the same IDs in
 * block_table_host, checked to lie in the pool) and streamed to the host
 * through two caller buffers of staging_bytes each (at least two pages;
 * 16-byte aligned): staging_dev (device memory) and staging (pinned host
 * memory).  Each is used as two halves in turn: a kernel packs pages into a
 * device half, a copy moves them to the host half, and the host writes the
 * other half meanwhile, so the memory used is those buffers, whatever
 * n_pos is (no copy of the cache is made).  The file is written as
 * path + ".tmp" and renamed to path once complete and flushed (fsync), so
 * path holds either a whole snapshot or what it held before; on failure the
 * temporary file is removed.  Format: safetensors (8-byte little-endian
 * header length, JSON header, data), one U8 tensor "layer<l>" of shape
 * [ceil(n_pos / page_size)][page_bytes] per layer, the layout and n_pos in
 * the header's metadata; whole pages are saved (slots past n_pos as they
 * are).  Synchronous: returns once the file is published.  The request
 * keeps its pages, which must not change or be released until the call
 * returns.  JF_ERR_INVALID for staging buffers of the wrong kind; JF_ERR_IO
 * on file errors, with errno's text in jf_last_error. */
jf_status jf_snapshot_save(const char* path, const jf_kv_layout* layout,
                           const jf_kv_pool_ptrs* pools, int32_t n_layers,
                           const int32_t* block_table, const int32_t* block_table_host,
                           int32_t max_pages, int32_t n_pos, void* staging_dev,
                           void* staging, size_t staging_bytes, hipStream_t stream);

/* Restore a snapshot written by jf_snapshot_save with the same layout and
 * layer count into the pages of a request's table (block_table device,
 * block_table_host the same IDs; its first ceil(n_pos / page_size) entries
 * must be distinct pages of the pool, reserved by the caller), writing the
 * packed runs straight into those pages: pieces of the file are read into
 * the pinned staging halves in turn, copied to the device halves and
 * unpacked by a kernel while the next piece is read.  *n_pos_out receives
 * the snapshot's position count.  Synchronous.  JF_ERR_INVALID if the file
 * is not such a snapshot (header, layout, layer count or size differ), the
 * table is too short or lists a page twice, or a staging buffer is of the
 * wrong kind; JF_ERR_IO on read errors. */
jf_status jf_snapshot_restore(const char* path, const jf_kv_layout* layout,
                              const jf_kv_pool_ptrs* pools, int32_t n_layers,
                              const int32_t* block_table, const int32_t* block_table_host,
                              int32_t max_pages, void* staging_dev, void* staging,
                              size_t staging_bytes, int32_t* n_pos_out, hipStream_t stream);

/* ---------------------------------------------------------------- TQ4
 * The paper's own 4-bit format (Sec. 3.1, eq. codec; Appendix A, Table
 * codec): a 256-element vector x is stored as the fp16 norm of x and 256
 * 4-bit indices z, where z_i indexes the one of 16 shared centroids c
 * (ascending) nearest to coordinate i of the rotated unit vector
 * y = H_256 S x / (16 |x|) (H_256 the unnormalised Sylvester Hadamard matrix,
 * S = diag(signs)).  Reconstruction: x_hat = norm * S H_256 c[z] / 16.
 *
 * Pool (per layer, per K or V; caller-owned device memory), head-major
 * pages like the affine pool:
 *   words  u32  [num_pages][num_kv_heads][page_size][32]  element 8w + k of
 *               a vector in bits 4k..4k+3 of word w
 *   norms  fp16 [num_pages][num_kv_heads][page_size]
 * Only page_size, num_kv_heads, head_dim (256) and num_pages of the layout
 * are used; group_size is ignored. */
jf_status jf_tq4_pool_bytes(const jf_kv_layout* layout, size_t* words_bytes,
                            size_t* norms_bytes);

/* Encode-and-append total_tok rows of K or V (one call per tensor, each
 * with its own signs) into a TQ4 pool, async on `stream`, one kernel.
 *   x            fp16 [total_tok][num_kv_heads][256] (device, 8-byte aligned)
 *   signs        fp32 [256] (device, 16-byte aligned), each +1 or -1
 *   centroids    fp32 [16] (device), ascending
 *   cu_tok, start_pos, block_tables, B, max_pages: as in
 *                jf_kv_quantize_append (row i of request b goes to logical
 *                position start_pos[b] + i; rows whose position falls outside
 *                the table or whose page ID is outside [0, num_pages) are
 *                not written)
 * Norm: the float32 Euclidean norm, rounded to fp16 (+inf when the norm
 * exceeds the fp16 range, i.e. |x| >= 65520; such vectors are out of range
 * for decode).  Index of a coordinate:
 * the number of thresholds (c_j + c_{j+1}) / 2 (float32) it strictly exceeds.
 * A zero vector gets norm 0 and the indices of coordinate 0.
 * Errors: NULL or misaligned pointers, B or max_pages <= 0, total_tok < 0,
 * max_pages * page_size above INT32_MAX -> JF_ERR_INVALID; head_dim != 256
 * or total_tok * num_kv_heads above INT32_MAX -> JF_ERR_UNSUPPORTED; no
 * launch on error. */
jf_status jf_tq4_encode_append(const jf_kv_layout* layout, void* words,
                               void* norms, const void* x, const float* signs,
                               const float* centroids, const int32_t* cu_tok,
                               const int32_t* start_pos,
                               const int32_t* block_tables, int32_t B,
                               int32_t max_pages, int32_t total_tok,
                               hipStream_t stream);

/* Single-query decode attention over TQ4 pages (Sec. 3.1, eq. codec: the
 * page-native decode reads the packed indices and norms where they are
 * stored).  Query head h reads KV head h / (num_q_heads / Hkv); request b
 * attends to its logical positions 0..seq_lens[b]-1 through its page table.
 * Computed without reconstructing any vector: the query is rotated once
 * (q' = H S_k q / 16), each position's logit is softmax_scale * norm_k *
 * (q' . c[z_k]), the weighted sum u = sum_t p_t norm_v c[z_v] is kept in the
 * rotated space, and the output is S_v H u / (16 sum_t p_t).
 *   k_words, v_words  u32 [NP][Hkv][P][32] (TQ4 pool layout above), 16-byte
 *                     aligned; k_norms, v_norms fp16 [NP][Hkv][P], 16-byte
 *                     aligned
 *   k_signs, v_signs  fp32 [256] (device): the sign diagonals the vectors
 *                     were encoded with; centroids fp32 [16] (device)
 *   q, out            fp16 [B][num_q_heads][256] (device)
 *   block_tables, max_pages, seq_lens, softmax_scale, max_splits,
 *   workspace         as in jf_decode_attn_q4, the workspace sized by
 *                     jf_decode_workspace_bytes(B, num_q_heads, 256,
 *                     max_splits) (same zero-counter rules)
 * Arithmetic: centroids rounded to fp16 once, q' as an fp16 high plus low
 * part, products on fp16 matrix cores with fp32 accumulation.  A norm that
 * overflowed fp16 at encode time (|x| above 65504) is +inf and makes the
 * outputs of every query reading that position non-finite.
 * Errors: head_dim != 256, page_size not a multiple of 32 or more than 16
 * query heads per KV head -> JF_ERR_UNSUPPORTED; NULL or misaligned
 * pointers, bad sizes, a short workspace or a non-finite scale ->
 * JF_ERR_INVALID; no launch on error. */
jf_status jf_tq4_decode_attn(const jf_kv_layout* layout, const void* k_words,
                             const void* k_norms, const void* v_words,
                             const void* v_norms, const float* k_signs,
                             const float* v_signs, const float* centroids,
                             const void* q, int32_t B, int32_t num_q_heads,
                             const int32_t* block_tables, int32_t max_pages,
                             const int32_t* seq_lens, float softmax_scale,
                             int32_t max_splits, void* workspace,
                             size_t workspace_bytes, void* out,
                             hipStream_t stream);

/* TQ4 page -> operand reconstruction (Appendix A, Table codec: page lookup,
 * index unpacking, centroid lookup, inverse rotation and norm restoration
 * in one kernel; Sec. 3.1, eq. groupattention): x_hat = norm * S H_256
 * c[z] / 16 for KV heads kv0 .. kv0 + num_heads - 1 at logical positions
 * 0 .. n_pos - 1 of one request, as contiguous fp16 k_out, v_out
 * [num_heads][n_pos][256] (device, 8-byte aligned).  Arithmetic in fp32
 * (centroids as given, the transform's sums, then signs and norm / 16),
 * rounded once to fp16.  Pool, signs and centroids as in
 * jf_tq4_decode_attn; block_table int32 [max_pages] (device).  A page ID
 * outside [0, num_pages) gives zero vectors. */
jf_status jf_tq4_reconstruct(const jf_kv_layout* layout, const void* k_words,
                             const void* k_norms, const void* v_words,
                             const void* v_norms, const float* k_signs,
                             const float* v_signs, const float* centroids,
                             const int32_t* block_table, int32_t max_pages,
                             int32_t n_pos, int32_t kv0, int32_t num_heads,
                             void* k_out, void* v_out, hipStream_t stream);

/* ---------------------------------------------------------------- KV8
 * An 8-bit cache beside the 4-bit ones, for models that do not bear 4 bits,
 * and what shortens a cache: the attention weights that its positions receive,
 * and eviction by them.  Query heads share KV heads and requests own page
 * tables as everywhere in this library.
 *
 * Stored element: c * 2^e, c an e4m3 code (OCP: 4 exponent and 3 mantissa
 * bits, largest 448, no infinity), e one exponent for each (page, KV head,
 * block of group_size consecutive positions), the same for K and V apart.
 * jf_kv_layout.group_size counts POSITIONS here: 16, 32, 64 or 128, a divisor of
 * page_size.  head_dim is 64, 128 or 256, page_size a multiple of 64 up to 4096.
 * Pool (jf_kv_pool_ptrs; codes 16-byte aligned, k_meta and v_meta hold the
 * exponent bytes):
 *   k_codes  uint8 [NP][Hkv][P][d]
 *   v_codes  uint8 [NP][Hkv][P/16][d/64][4][16][4][4]: token t, dim c of a
 *            page's head lie at [t/16][c/64][t%16/4][c%64/4][c%4][t%4]
 *   k_meta, v_meta  uint8 [NP][Hkv][P/group_size]  e + 127
 * Quantizer (bit-exact contract), per block: amax over the finite elements of
 * the rows; e = the least exponent >= -126 with amax <= 448 * 2^e (a block of
 * zeros: -126); c = x * 2^-e rounded to the nearest e4m3 value, ties to even.
 * Inputs must be finite; an infinity is stored as the block's largest value
 * (+-448 * 2^e) and a NaN as +0, so that no stored code is a NaN.
 *
 * Types: k_new, v_new, q and out are fp16 (JF_F16) or bf16 (JF_BF16), one type
 * per call; products run on the matrix cores with fp32 accumulation, codes
 * enter them exactly, softmax statistics and sums are fp32.  Beside the values
 * (decode and chunk attention) a probability is rounded to fp16: by up to 2^-11 of
 * itself, or 2^-25 of its row's largest where that is more.  The sum that divides
 * them, lse and added weights are formed before that rounding.
 * Limits of the attention calls, in magnitude: q finite, with a sum over a head's dims
 * below 2^90; softmax_scale * k below 2^110 and softmax_scale * q . k below 2^126;
 * v below 2^90.  (fp16 rows and an ordinary scale are far from them.)  Next to values
 * of its head that are 2^80 times as large, a value may count as 0.
 * Outputs must overlap neither inputs nor workspaces.  Every function
 * returns JF_ERR_UNSUPPORTED for a geometry, type or size that is not
 * implemented and JF_ERR_INVALID for NULL or misaligned pointers, bad sizes, a
 * short workspace or a scale that is not finite or not below 2^126 in magnitude;
 * nothing is launched then. */
typedef enum { JF_F16 = 0, JF_BF16 = 1 } jf_dtype;

/* Bytes of one codes array and of one exponent array (the same for K and V). */
jf_status jf_kv8_pool_bytes(const jf_kv_layout* layout, size_t* codes_bytes,
                            size_t* exps_bytes);

/* Quantize rows of K and V into their pages.  k_new, v_new: [total_tok][Hkv][d]
 * (device, 16-byte aligned); cu_tok, start_pos, block_tables, B, max_pages as in
 * jf_kv_quantize_append: rows whose position is negative or beyond the table, or
 * whose page ID is outside [0, num_pages), are skipped.
 * A block that holds positions before request b's first new row (start_pos[b]
 * inside a block) keeps them: its exponent becomes the larger of the stored one
 * and the new rows' one, and if that raises it, the stored codes of those earlier
 * positions are rescaled (exact but for codes that become subnormal, which are
 * rounded once more).  Slots behind the last new row are left as they are.
 * Rows of one call must not share a position; pages must not be shared. */
jf_status jf_kv8_append(const jf_kv_layout* layout, const jf_kv_pool_ptrs* pool,
                        int32_t dtype, const void* k_new, const void* v_new,
                        const int32_t* cu_tok, const int32_t* start_pos,
                        const int32_t* block_tables, int32_t B, int32_t max_pages,
                        int32_t total_tok, hipStream_t stream);

/* Decode attention: the last num_queries (1..4) positions of request b, already
 * appended, are its query tokens; token k sees the positions 0 .. seq_lens[b] -
 * num_queries + k.  Lengths are cut to the table's capacity; a token that sees
 * nothing gets a zero row.
 *   q, out      [B][num_queries][num_q_heads][d] (device, 16-byte aligned)
 *   max_splits  cap on partials per request and KV head (1..1024).  A request's
 *               output depends on neither the batch nor the other requests.
 *   workspace   16-byte aligned device scratch of at least
 *               jf_kv8_decode_workspace_bytes().  Its first 262,144 bytes must be
 *               zero before the first call; every call that completes leaves them
 *               zero (the workspace of jf_decode_attn_q4 has the same rule, and
 *               one that is large enough serves both).  Calls that may overlap in
 *               time, replays of graphs among them, must not share one.
 *   weights     NULL, or fp32 (device): weights[(b * Hkv + kv) * weights_stride
 *               + t] grows by the sum, over the call's tokens and the query heads
 *               of kv, of the attention weight of position t < seq_lens[b].
 *               Entries from seq_lens[b] on are left as they are.
 *               weights_stride >= max_pages * page_size; the workspace is then
 *               sized with weight_pages = max_pages (else 0), 4 bytes per score.
 * Positions on a page ID outside [0, num_pages) do not contribute.
 * B <= 65,535 and B * num_q_heads * num_queries <= 65,536. */
jf_status jf_kv8_decode_workspace_bytes(const jf_kv_layout* layout, int32_t B,
                                        int32_t num_queries, int32_t num_q_heads,
                                        int32_t max_splits, int32_t weight_pages,
                                        size_t* bytes);
jf_status jf_kv8_decode_attn(const jf_kv_layout* layout,
                             const jf_kv_pool_ptrs* pool, int32_t dtype,
                             const void* q, int32_t B, int32_t num_queries,
                             int32_t num_q_heads, const int32_t* block_tables,
                             int32_t max_pages, const int32_t* seq_lens,
                             float softmax_scale, int32_t max_splits,
                             void* workspace, size_t workspace_bytes, void* out,
                             float* weights, int64_t weights_stride,
                             hipStream_t stream);

/* Chunk attention of one request: rows 0 .. T-1 sit at positions prefix_len .. +
 * T-1, which are already in the cache (append first, unlike jf_prefill_attn_q4),
 * and attend causally to the positions 0 .. prefix_len + i, all read from the
 * pages.
 *   q, out     [T][num_q_heads][d] (device, 16-byte aligned)
 *   lse        NULL, or fp32 [T][num_q_heads] (device): the natural logarithm of
 *              the sum of exp(softmax_scale * q . k) over the positions seen
 *              (-inf where there is none, for which out is zero)
 *   workspace  NULL, or 16-byte aligned device scratch of at least
 *              jf_kv8_prefill_workspace_bytes() (which may be 0): lets a chunk of
 *              few rows share its keys among more blocks.  Its contents do not
 *              matter.  Calls that may overlap in time must not share one.
 *              Results with and without it are the same up to the order of sums.
 *              The bytes belong to one T and prefix_len and do not grow with them
 *              (64 rows, 32/8 heads of 128: 34.6 MB after 30,000 positions, 33.5
 *              after 65,536; 2,048 rows after as many: none).  One workspace for many
 *              calls has the largest of their sizes; a call that needs more than
 *              there is can be given NULL, and is refused with less.
 * Positions on a page ID outside [0, num_pages) do not contribute. */
jf_status jf_kv8_prefill_workspace_bytes(const jf_kv_layout* layout, int32_t T,
                                         int32_t num_q_heads, int32_t prefix_len,
                                         size_t* bytes);
jf_status jf_kv8_prefill_attn(const jf_kv_layout* layout,
                              const jf_kv_pool_ptrs* pool, int32_t dtype,
                              const void* q, int32_t T, int32_t num_q_heads,
                              const int32_t* block_table, int32_t max_pages,
                              int32_t prefix_len, float softmax_scale,
                              void* workspace, size_t workspace_bytes, void* out,
                              float* lse, hipStream_t stream);

/* Attention weights of a chunk's rows, added up per position: weights[kv *
 * weights_stride + t] grows by the sum, over rows i and the query heads h of kv
 * with t <= prefix_len + i, of exp(softmax_scale * q_ih . k_t - lse_ih).  q and lse
 * as of jf_kv8_prefill_attn; for the last rows of a chunk only (an observation
 * window) pass their q, lse and prefix_len.  Entries from prefix_len + T on, and
 * those of positions on a page ID outside [0, num_pages), are left as they are.
 * weights: fp32 (device), weights_stride >= prefix_len + T.  The sums' order is
 * fixed: the same inputs give the same bits. */
jf_status jf_kv8_attn_weights(const jf_kv_layout* layout,
                              const jf_kv_pool_ptrs* pool, int32_t dtype,
                              const void* q, const float* lse, int32_t T,
                              int32_t num_q_heads, const int32_t* block_table,
                              int32_t max_pages, int32_t prefix_len,
                              float softmax_scale, float* weights,
                              int64_t weights_stride, hipStream_t stream);

/* Eviction by accumulated weight.  For each request b and KV head, m =
 * min(seq_lens[b], keep) positions stay: the last min(recent, seq_lens[b]) and,
 * of the others, those of the largest weights (ties: the lowest positions; a NaN
 * counts as larger than any number).  They are moved, in their order, to the
 * positions 0 .. m - 1 of dst_tables' pages, whose blocks get exponents of their
 * own (a moved code changes by a power of two; exact but for codes that become
 * subnormal).  The caller goes on with dst_tables and length m, and returns the
 * old pages.
 *   weights       fp32 [B][Hkv][weights_stride] (device), as added up by the
 *                 calls above; weights_stride >= max_pages * page_size
 *   keep, recent  1 <= keep < 2^30, 0 <= recent <= keep
 *   dst_tables    int32 [B][dst_max_pages] (device), keep <= dst_max_pages *
 *                 page_size; its pages must be none of the source pages, and
 *                 distinct.  Positions on a page ID outside [0, num_pages) are not
 *                 written (source: they are moved as zeros).
 *   workspace     16-byte aligned device scratch of at least
 *                 jf_kv8_evict_workspace_bytes() (may be 0, then NULL will do);
 *                 its contents do not matter.  Calls that may overlap in time
 *                 must not share one.
 *   kept          int32 [B][Hkv][keep]: the positions that stay, ascending, then -1
 *   kept_weights  fp32 [B][Hkv][keep]: their weights, then 0.  Calls that go on adding
 *                 to them take rows of at least the new tables' capacity: copy them
 *                 to the start of such rows, zeros behind.
 * Slots behind position m - 1 are left as they are. */
jf_status jf_kv8_evict_workspace_bytes(const jf_kv_layout* layout, int32_t B,
                                       int32_t max_pages, int32_t keep,
                                       size_t* bytes);
jf_status jf_kv8_evict(const jf_kv_layout* layout, const jf_kv_pool_ptrs* pool,
                       int32_t B, const int32_t* block_tables, int32_t max_pages,
                       const int32_t* seq_lens, const float* weights,
                       int64_t weights_stride, int32_t keep, int32_t recent,
                       const int32_t* dst_tables, int32_t dst_max_pages,
                       void* workspace, size_t workspace_bytes, int32_t* kept,
                       float* kept_weights, hipStream_t stream);

/* Decode attention of a batch whose requests share prefixes: as jf_kv8_decode_attn
 * (the same queries, masks, types, roundings and limits), with the positions that a
 * group's requests have in common read once for all of them.  Attention weights are not
 * added up here: a program that evicts by them takes them from jf_kv8_decode_attn or
 * jf_kv8_attn_weights.
 *   group_start  int32 [num_groups + 1] (device): requests group_start[g] ..
 *                group_start[g + 1] - 1 are group g; ascending from 0 to B (otherwise
 *                every request is computed by itself).  Groups of one request, or none,
 *                are allowed.
 *   shared_lens  int32 [num_groups] (device): the first shared_lens[g] positions of
 *                group g's requests hold the same keys and values.  They are read
 *                through the table of the group's first request, and cut to its
 *                length; what other tables hold for whole pages of them is not looked
 *                at.  Any length will do, in the middle of a page too, 0 for none.
 *   workspace    16-byte aligned device scratch of at least
 *                jf_kv8_shared_workspace_bytes(); its contents do not matter before
 *                the call nor after it.  Calls that may overlap in time, replays of
 *                graphs among them, must not share one.
 *   lse          NULL, or fp32 [B][num_queries][num_q_heads] (device): the natural
 *                logarithm of the sum of exp(softmax_scale * q . k) over the positions
 *                seen (-inf where there is none, for which out is zero)
 * Lengths and groups are read on the device: a captured call can be replayed with
 * others.  The kernels are chosen on the host by B, the heads and max_pages, an upper
 * bound of what is read: tables far wider than the requests are long cost time (64
 * requests over 4,096 positions, 32/8 heads of 128: 37 us, or 58).  Two calls with the same inputs give the same bits; a request's results in
 * another batch are the same up to the order of sums.  B <= 65,535,
 * B * num_q_heads * num_queries <= 65,536, 1 <= num_groups <= B. */
jf_status jf_kv8_shared_workspace_bytes(const jf_kv_layout* layout, int32_t B,
                                        int32_t num_groups, int32_t num_queries,
                                        int32_t num_q_heads, size_t* bytes);
jf_status jf_kv8_shared_attn(const jf_kv_layout* layout,
                             const jf_kv_pool_ptrs* pool, int32_t dtype,
                             const void* q, int32_t B, int32_t num_queries,
                             int32_t num_q_heads, const int32_t* block_tables,
                             int32_t max_pages, const int32_t* seq_lens,
                             const int32_t* group_start, const int32_t* shared_lens,
                             int32_t num_groups, float softmax_scale, void* workspace,
                             size_t workspace_bytes, void* out, float* lse,
                             hipStream_t stream);

/* ---------------------------------------------------- rotary positions
 * Rows of queries and keys rotated by their tokens' positions, as the models whose
 * caches this library keeps do before attention.  Of a head's dims the first rot_dim
 * are rotated in rot_dim / 2 pairs, pair i of a token at position p by the angle
 * p * f_i; the others stay:
 *   (y1, y2) = (x1 c - x2 s, x2 c + x1 s),  c = m cos(p f_i),  s = m sin(p f_i)
 * A pair is dims i and i + rot_dim / 2 (JF_ROPE_HALVES) or 2 i and 2 i + 1
 * (JF_ROPE_PAIRS).  c and s are fp32 values of a table that a step forms once for all
 * of its layers (and a training program once); each product and sum is rounded in
 * fp32, the result once to the rows' type (JF_F16 or JF_BF16). */
typedef enum { JF_ROPE_HALVES = 0, JF_ROPE_PAIRS = 1 } jf_rope_order;

/* How frequencies f_i = base^(-2 i / rot_dim) are changed for contexts `factor` times
 * as long as the model's own (original_len positions):
 *   JF_ROPE_PLAIN    not at all
 *   JF_ROPE_LINEAR   f_i / factor (position interpolation)
 *   JF_ROPE_BASE     base * factor^(rot_dim / (rot_dim - 2)) in base's place: the
 *                    fastest pair stays, the slowest is divided by factor
 *   JF_ROPE_PARTS    pairs of more than `fast` turns in original_len positions stay,
 *                    those of fewer than `slow` are divided by factor, between them
 *                    lies a ramp over the pairs' numbers:
 *                    i(r) = rot_dim ln(original_len / (2 pi r)) / (2 ln base), the ramp
 *                    from floor(i(fast)), at least 0, to ceil(i(slow)), at most
 *                    rot_dim - 1 (without length where all pairs lie on one side of
 *                    it: they stay, or from ceil(i(slow)) on are divided);
 *                    m = 0.1 ln(factor) + 1 (factor <= 1: 1).  The parts and the
 *                    magnitude are those of "YaRN" (arXiv 2309.00071), whose own ramp
 *                    is linear in a pair's turns, and not in its number as it is here
 *                    and in models that are published with this scaling */
typedef enum {
  JF_ROPE_PLAIN = 0,
  JF_ROPE_LINEAR = 1,
  JF_ROPE_BASE = 2,
  JF_ROPE_PARTS = 3
} jf_rope_scaling;

/* The frequencies and the magnitude m (1 but for JF_ROPE_PARTS), on the host.  Formed
 * in 64 bits, rounded once to fp32.  inv_freq: float [rot_dim / 2] (host);
 * magnitude: float (host).  base > 1; factor > 0 (unless PLAIN); for PARTS
 * original_len >= 1 and fast > slow > 0.  Arguments a scaling does not use are not
 * looked at.  rot_dim even, 2 .. 65536 (BASE: from 4 on). */
jf_status jf_rope_frequencies(int32_t rot_dim, double base, int32_t scaling, double factor,
                              int32_t original_len, double fast, double slow, float* inv_freq,
                              float* magnitude);

/* table[j][i] = (c, s) of position positions[j] and frequency inv_freq[i]:
 *   positions  int32 [n] (device), any values
 *   inv_freq   fp32 [rot_dim / 2] (device), magnitudes that keep |p f| below 2^40
 *   table      fp32 [n][rot_dim / 2][2] (device, 8-byte aligned)
 * The angle is exact (64 bits and a rest), c and s are rounded once to fp32. */
jf_status jf_rope_table(const int32_t* positions, int32_t n, const float* inv_freq,
                        int32_t rot_dim, float magnitude, float* table, hipStream_t stream);

/* The angles of a call's tokens: token j takes row rows[j] of the table (int32
 * [total_tok], device; an entry outside the table is cut to its first or last row), or
 * row j where rows is NULL (the table then has at least total_tok rows). */
typedef struct {
  const float* table;  /* [table_rows][rot_dim / 2][2], device, 8-byte aligned */
  const int32_t* rows;
  int32_t table_rows;
  int32_t rot_dim;     /* even */
  int32_t order;       /* jf_rope_order */
} jf_rope;

/* Rotate rows of queries and of keys in one launch; transpose != 0: s with the other
 * sign, which turns back (m = 1) and takes gradients of the outputs to gradients of
 * the inputs.
 *   q, k   [total_tok][heads][head_dim] (device), a token's heads one after the other,
 *          q_stride (k_stride) elements from one token to the next: rows of their own,
 *          or part of a wider projection's rows.  num_q_heads = 0 or num_k_heads = 0:
 *          none (the pointers are not looked at).
 *   q_out, k_out   the same shape and strides of their own.  An output may be its
 *          input (same pointer and stride); otherwise the memory of outputs must not
 *          overlap that of inputs or of the other output.
 * head_dim even and at most 65536, rot_dim <= head_dim, strides at least heads *
 * head_dim where total_tok > 1 and at most 2^31.  Addresses aligned to an element are enough; 16 bytes,
 * with sizes and strides of multiples of 16 and 8 elements, are fastest. */
jf_status jf_rope_rotate(const jf_rope* rope, int32_t dtype, int32_t head_dim, int32_t transpose,
                         const void* q, int64_t q_stride, void* q_out, int64_t q_out_stride,
                         int32_t num_q_heads, const void* k, int64_t k_stride, void* k_out,
                         int64_t k_out_stride, int32_t num_k_heads, int32_t total_tok,
                         hipStream_t stream);

/* jf_kv8_append of keys that are rotated on the way, and the rotation of the same
 * tokens' queries, in one launch: the cache and q_out are, bit for bit, those of
 * jf_rope_rotate followed by jf_kv8_append.
 *   rope      as above, rot_dim a multiple of 16 and at most the layout's head_dim
 *   k_new, v_new  [total_tok][Hkv][d] (device, 16-byte aligned), k_stride and
 *             v_stride elements from one token to the next (multiples of 8, at least
 *             Hkv * d where total_tok > 1, at most 2^31)
 *   q, q_out  NULL, or [total_tok][num_q_heads][d] (device, 16-byte aligned), q with
 *             q_stride as above, q_out without gaps; q_out may be q where q has none
 * The positions that turn a key need not be the cache's (after an eviction they are
 * not).  Other arguments and rules as jf_kv8_append; every token's query is rotated,
 * also those whose keys are skipped. */
jf_status jf_kv8_rope_append(const jf_kv_layout* layout, const jf_kv_pool_ptrs* pool,
                             int32_t dtype, const jf_rope* rope, const void* k_new,
                             int64_t k_stride, const void* v_new, int64_t v_stride, const void* q,
                             int64_t q_stride, void* q_out, int32_t num_q_heads,
                             const int32_t* cu_tok, const int32_t* start_pos,
                             const int32_t* block_tables, int32_t B, int32_t max_pages,
                             int32_t total_tok, hipStream_t stream);

#ifdef __cplusplus
}
#endif
#endif /* JFKV_H */
