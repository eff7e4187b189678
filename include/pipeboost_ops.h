/*
 * pipeboost_ops.h -- kernel-level entry points of libpipeboost.so.
 *
 * Each call runs one kernel of the prefill (plus its split-K reduce where the
 * launcher splits) on caller-provided device buffers, on the given stream,
 * asynchronously.  They exist to test every kernel against the CPU oracle's
 * component functions and to time kernels in isolation; the model API in
 * pipeboost.h is the product path.  The last section is for programs that run
 * decode steps of their own over a cache of pages.  All pointers are device pointers, all
 * matrices row-major with the reduction dimension contiguous; "dt" is
 * bfloat16 (dtype 0) or IEEE binary16 (dtype 1).  Every call returns a
 * pb_status (PB_EINVAL for unsupported shapes, PB_EHIP for launch failures,
 * message in pb_last_error()).
 */
#ifndef PIPEBOOST_OPS_H
#define PIPEBOOST_OPS_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

/* Projection GEMM Y = X W^T (fp32 accumulate) with an epilogue
 * (Section 2.1: the decoder's linear layers; bias as in OPT):
 *   epi 0: C = dt((Y + bias) * (n < qcols ? qscale : 1))   (q, k, v projection)
 *   epi 1: C = dt(max(Y + bias, 0))                        (fc1 with ReLU)
 *   epi 2: R += Y + bias, R fp32 [M, N] (ldr = N)           (o and fc2, residual)
 * X [M, K] dt, W [N, K] dt, bias [N] dt, C [M, N] dt (ldc = N).  Requires
 * N % 64 == 0 and K % 64 == 0.  workspace (fp32 scratch for split-K partials,
 * may be NULL) of workspace_bytes. */
int pb_op_gemm(int32_t dtype, int32_t epi, const void* X, const void* W, const void* bias,
               void* C, float* R, int32_t M, int32_t N, int32_t K, float qscale, int32_t qcols,
               void* workspace, size_t workspace_bytes, void* stream);

/* pb_op_gemm with the unmerged LoRA expand folded into the same accumulation
 * as extra K tiles (Section 2.1: the adapter adds s (x A) B on top of the
 * fixed W; Section 4.2.2: sequences of one batch may use different adapters):
 *   Y[m, n] = X[m] . W[n] + Z[m, g zs .. g zs + K2) . W2[n]   if bit g of group_mask
 *           = X[m] . W[n]                                     otherwise,
 * with g = n / group (the output group: q, k, v of a fused projection),
 * then the epilogue of pb_op_gemm.  Z [M, ldz] dt holds each row's scaled
 * shrink s (x A_slot) in its adapter slot's columns of every group block
 * (zeros in the other slots' columns, so rows of different adapters, or none,
 * share the launch); W2 [N, K2] dt holds the B matrices of all slots side by
 * side.  K2 % 64 == 0, group % 256 == 0; other requirements and the workspace
 * as pb_op_gemm. */
int pb_op_gemm_lora(int32_t dtype, int32_t epi, const void* X, const void* W, const void* bias, void* C,
                    float* R, int32_t M, int32_t N, int32_t K, const void* Z, int32_t ldz, int32_t zs,
                    const void* W2, int32_t K2, int32_t group, uint32_t group_mask, float qscale,
                    int32_t qcols, void* workspace, size_t workspace_bytes, void* stream);

/* pb_op_gemm for callers that cannot allocate (code under HIP graph capture,
 * tight serving loops, harnesses that forbid hipMalloc): the same operands,
 * epilogues and kernels, with the split-K partials in a 64 MiB device array
 * of the library instead of a caller workspace.  The call allocates nothing
 * (no hipMalloc, hipFree or allocating library routine); the array is part
 * of the library's code object, one copy per GPU, held until the process
 * ends.  The result is bit-identical to pb_op_gemm given a 64 MiB workspace.
 * Products are limited to M * N * 4 <= 64 MiB (PB_EINVAL above it: use
 * pb_op_gemm).  The array of the current device is used, so `stream` must
 * belong to that device.  Every call on a GPU shares that GPU's array: calls
 * that overlap on one GPU (other streams or threads) race. */
int pb_op_gemm_noalloc(int32_t dtype, int32_t epi, const void* X, const void* W, const void* bias,
                       void* C, float* R, int32_t M, int32_t N, int32_t K, float qscale,
                       int32_t qcols, void* stream);

/* Causal multi-head self-attention over B sequences of T tokens (Section 2.1:
 * prefill self-attention; token j attends to tokens 0..j).  qkv [B*T, 3*H*hd]
 * dt with q already divided by sqrt(hd), out [B*T, H*hd] dt; hd in {64, 128}. */
int pb_op_attention(int32_t dtype, const void* qkv, void* out, int32_t B, int32_t T,
                    int32_t H, int32_t hd, void* stream);

/* LayerNorm of rows of an fp32 matrix x [rows, d]: out = LN(x) * g + b with
 * fp32 statistics (biased variance); g, b [d] dt; out [rows, d] dt, or fp32
 * when out_f32 != 0.  d % 4 == 0, d <= 16384. */
int pb_op_layernorm(int32_t dtype, const float* x, const void* g, const void* b, void* out,
                    int32_t out_f32, int32_t rows, int32_t d, float eps, void* stream);

/* ---- a cache of pages, and beam search over it ----------------------------
 *
 * One decode step of sequences of any lengths, on caller-provided device
 * buffers: pb_op_page_fork orders the rows' pages after their parents and makes
 * room for the new tokens; per layer, pb_op_kv_append writes the new tokens'
 * keys and values (after a prefill: the prompts') and pb_op_paged_attention
 * attends to the pages; pb_op_beam_select picks the next tokens and parents.
 * Every call is a fixed sequence of kernels that reads lengths, tables and
 * parents on the device, so a step is captured into a HIP graph once and
 * replayed as the sequences grow; nothing is allocated.  Device tensors of
 * int32 are 4-byte aligned, a workspace 16-byte aligned.  A workspace carries
 * nothing from one call to the next: calls that run one after another on a
 * stream may share one (two recorded graphs too, if their replays do not
 * overlap), calls that may overlap need one each.  Every buffer and the stream
 * belong to the current device. */

/* Pages of one layer.  Element j of token t of head h, keys (c = 0) or values
 * (c = 1), of page i is at
 *   base + i page_stride + c v_offset + h head_stride + t token_stride + j,
 * strides in elements of dt, multiples of 8 and at least head_dim (that of a
 * dimension of size 1 is not used), token_stride below 2^31; base 16-byte aligned.  head_dim is 64 or 128,
 * page_size 1..4096 tokens, at most 2^30 pages.  Both a page that holds its tokens as the model's
 * cache rows [k | v] (token_stride 2 Hkv hd, v_offset Hkv hd, head_stride hd)
 * and one that holds each head's tokens in a row fit.  A page table row holds the
 * page of tokens 0 .. page_size-1, then the next, ...: int32 [rows][width]. */
typedef struct {
    void* base;
    int64_t page_stride, v_offset, head_stride, token_stride;
    int32_t n_pages, page_size, n_kv_heads, head_dim;
} pb_kv_pool;

/* Keys and values of new tokens into the pages of their sequences: sequence s
 * gains tokens start[s] .. lens[s]-1, token start[s] + i from row row0[s] + i of k
 * and v ([n_rows][Hkv hd] dt with row strides ld_k, ld_v in elements, multiples
 * of 8; rows of a fused q, k, v projection fit).  row0 NULL: sequence s's rows
 * start at s max_rows (a padded batch).  max_rows: at most so many tokens per
 * sequence are written (it sizes the launch).  start[s] >= lens[s] or start[s] <
 * 0: none.  A token past the table's width, on a page id outside the pool, or
 * of a row outside [0, n_rows) is not written; no other byte of the pool
 * changes.  Two sequences must not name the same token of a page. */
int pb_op_kv_append(int32_t dtype, const void* k, int64_t ld_k, const void* v, int64_t ld_v, int32_t n_rows,
                    const pb_kv_pool* pool, const int32_t* tables, int32_t width, int64_t ld_tables,
                    const int32_t* start, const int32_t* lens, const int32_t* row0, int32_t n_seqs,
                    int32_t max_rows, void* stream);

/* Attention of one new token per sequence: row s of q ([n_seqs] rows of n_heads hd
 * dt, row stride ld_q) attends to tokens 0 .. lens[s]-1 of its pages, or with
 * window > 0 to the last `window` of them:
 *   out[s, h] = sum_x softmax_x(scale q[s, h] . K[x, h / (n_heads / Hkv)]) V[x, ...].
 * The token's own key and value are in the pages already (pb_op_kv_append).
 * n_heads is a multiple of Hkv; ld_q and ld_out multiples of 8, q and out 16-byte
 * aligned.  lens[s] <= 0: zeros.  A row with a page id outside the pool, or past
 * the table's width, among the tokens it attends to: NaN (pages before the window
 * are not looked at).  Nothing past a sequence's last token is read.
 * shared != 0 says that rows next to each other share pages (beams of one prompt):
 * caches are used then for what otherwise streams past them; results are the same.
 * Scores, maxima, sums and products are fp32; probabilities enter the products with
 * V and their sum within 2^-21 (f16) or 2^-15 (bf16) of themselves.
 * workspace (may be NULL): fp32 partial results of the pieces that long
 * sequences are cut into, pb_op_paged_attention_workspace bytes; with a smaller one
 * they are not cut.  It must not overlap the other operands.  Tables hold at most 2^30
 * tokens a row; sequences x key/value heads (of more than 32 heads each: x
 * blocks of 32) stay below 2^24 - 8. */
int pb_op_paged_attention(int32_t dtype, const void* q, int64_t ld_q, const pb_kv_pool* pool,
                          const int32_t* tables, int32_t width, int64_t ld_tables, const int32_t* lens,
                          int32_t n_seqs, int32_t n_heads, float scale, int32_t window, int32_t shared,
                          void* out, int64_t ld_out, void* workspace, size_t workspace_bytes, void* stream);

/* Workspace bytes for n_seqs sequences of tables of `width` pages (0 for
 * arguments pb_op_paged_attention refuses). */
size_t pb_op_paged_attention_workspace(int32_t n_seqs, int32_t n_heads, const pb_kv_pool* pool, int32_t width);

/* Beam search's selection.  Row b W + w of logits (fp32, row stride ld_logits
 * elements) belongs to hypothesis w of prompt b, with log probability scores[b, w] so
 * far.  A live hypothesis (alive != 0) offers every token v at scores + log
 * softmax(logits)[v]; an ended one (alive = 0) itself, at its score, as token
 * `pad`.  The W best of each prompt, best first, ties to the lowest w V + v:
 *   out_scores, out_tokens; out_parents: the row b W + w each continues;
 *   out_alive: 0 if it had ended or its token is eos (eos -1: none ends).
 * Scores are formed and compared in 64 bits, from log sums of fp32 exponentials
 * (within 2^-18: of two rows' continuations that are nearer than that either may
 * come first).  Logits of -inf or NaN are no candidates and have no part in the
 * softmax, one of +inf counts as the largest float; a hypothesis whose score is not
 * finite offers nothing (a prompt's first step: scores 0, -inf, -inf, ...), and a
 * continuation whose score is below the lowest float is none.  Places that no
 * candidate takes: score -inf, token pad, parent -1, alive 0.  out_scores and
 * out_alive may be scores and alive.  1 <= W <= 32, 1 <= V <= 2^20, 0 <= pad < V;
 * workspace: pb_op_beam_select_workspace bytes (0 for refused sizes). */
int pb_op_beam_select(const float* logits, int64_t ld_logits, const float* scores, const int32_t* alive,
                      int32_t B, int32_t W, int32_t V, int32_t eos, int32_t pad, float* out_scores,
                      int32_t* out_tokens, int32_t* out_parents, int32_t* out_alive, void* workspace,
                      size_t workspace_bytes, void* stream);
size_t pb_op_beam_select_workspace(int32_t B, int32_t W, int32_t V);

/* Reorder, share, copy on write, grow and free: the page tables of out_rows rows
 * from those of in_rows rows.  Row r takes the pages of row parents[r] (outside
 * [0, in_rows): it holds nothing) and room for grow[r] more tokens:
 *   out_start[r] = lens[parents[r]], out_lens[r] = out_start[r] + max(grow[r], 0).
 * refs[i] counts every reference to page i, those of `tables` (of the first
 * ceil(lens / page_size) pages of each row) among them; a page of count 0 is
 * free.  In out_refs the references of `tables` are replaced by those of
 * out_tables, so pages that no row takes over become free.
 * A row that grows needs its last page to itself if it is partly filled: when
 * every reference to that page is such a row's, the lowest of them keeps it and
 * the others get a copy; if anything else refers to it, all do.  A copy holds the
 * page's tokens of this row, in each of the n_layers layers (layer l's pages
 * layer_stride elements after layer l-1's); the rest of the new page is left as
 * it was.  New pages are the free ones in ascending order, to rows in ascending
 * order (a row's copy first), pages freed by this very call among them.
 * short_of[0]: how many pages are missing; if any is, no row grows or copies
 * (out_lens = out_start).  short_of[1]: rows that would pass the table's width;
 * they do not grow.  Table entries past a row's pages are -1.
 * tables, out_tables: [rows][width], contiguous.  Outputs and workspace must not
 * overlap the inputs or each other.  grow = 0 keeps, parents = -1 frees, an empty row with grow = T is a new
 * prompt's.  At most 65535 rows, and rows x layers x pieces of 32 KB of a page below
 * 2^31; workspace: pb_op_page_fork_workspace bytes.  A refused call writes nothing. */
int pb_op_page_fork(int32_t dtype, const pb_kv_pool* pool, int32_t n_layers, int64_t layer_stride,
                    const int32_t* parents, int32_t out_rows, const int32_t* tables, int32_t width,
                    const int32_t* lens, int32_t in_rows, const int32_t* refs, const int32_t* grow,
                    int32_t* out_tables, int32_t* out_start, int32_t* out_lens, int32_t* out_refs,
                    int32_t* short_of, void* workspace, size_t workspace_bytes, void* stream);
size_t pb_op_page_fork_workspace(int32_t out_rows, int32_t n_pages);

#ifdef __cplusplus
}
#endif

#endif /* PIPEBOOST_OPS_H */
