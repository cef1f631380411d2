/*
 * pbd_ops.h -- single-kernel entry points of libpbd, for per-kernel parity tests and for
 * callers that want one step of the pass on its own.  Same conventions as pbd.h: device
 * pointers (d_), asynchronous on the given stream, caller-provided workspace, pbd_status
 * return; the message of the last failure of these calls on this thread comes from
 * pbd_op_last_error().
 */
#ifndef PBD_OPS_H
#define PBD_OPS_H

#include "pbd.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Workspace bytes pbd_op_linear needs for these sizes (0 if unsupported). */
size_t pbd_op_linear_workspace_bytes(int32_t M, int32_t K, int32_t N, int32_t r);

/* One block linear with the switchable LoRA-like delta of the paper's adapter (Appendix A.2:
 * rank r, scale alpha/r, on every projection):
 *     u = bf16(x A^T)                    [M, r]
 *     y = bf16(x W^T + scale * u B^T)    [M, N]   (fp32 accumulation, one final rounding)
 * d_x [M, K], d_w [N, K], d_a [r, K], d_b [N, r], d_y [M, N]: bf16, row-major, 16-byte aligned.
 * d_a == NULL or d_b == NULL (or r == 0) switches the delta off.  W and A are read in place; K is
 * summed in 256-wide slices in one fixed order, as in the decoder passes, so without the adapter a
 * row's result does not depend on M.  d_y may lie over an operand (one more copy of y).
 * Requirements: N % 128 == 0, K % 64 == 0, 1 <= M <= 4096, r <= 32.
 * The workspace (d_ws, >= pbd_op_linear_workspace_bytes, 1024-byte aligned) is scratch; its first
 * word is the kernel's status word, cleared by each call and read by pbd_op_status.
 * The return value covers argument checks and launches only: a bounded device wait that ran out
 * is reported by pbd_op_status(d_ws, ...) after the call (before the next call on d_ws). */
pbd_status pbd_op_linear(int32_t M, int32_t K, int32_t N, int32_t r, float scale, const void *d_x, const void *d_w,
                         const void *d_a, const void *d_b, void *d_y, void *d_ws, size_t ws_bytes, void *d_stream);

/* Bytes of the library's own device scratch behind pbd_op_linear_static, per device. */
#define PBD_OP_LINEAR_STATIC_SCRATCH_BYTES (16u << 20)

/* pbd_op_linear without a workspace.  This entry point has no counterpart in the paper: it is
 * an integration aid.  It computes exactly what pbd_op_linear computes, with the same kernels
 * and the same fixed-order sums, so for the same inputs the two give the same y.
 *
 * Who it is for: callers that cannot hand the library device memory.  For example a caller
 * that sits behind an interface which passes only its input and output tensors, a process whose
 * device memory is entirely owned by another allocator, or a loop that must not call cudaMalloc
 * or cudaFree because those calls can synchronise the device.  Such a caller gets a call that
 * never allocates or frees device memory (no cudaMalloc, cudaFree, stream-ordered or library
 * allocation of any kind).
 *
 * Where the scratch lives: a fixed array of PBD_OP_LINEAR_STATIC_SCRATCH_BYTES (16 MiB) in the
 * library's device code, one per device, created when the CUDA runtime loads that code on the
 * device.  Its address is looked up the first time this function is called with a device current
 * (also the time the kernels' attributes are set); make that first call on each device before
 * any stream capture begins.
 *
 * Size limit: the call needs 2048 + (N/128 + (r > 0)) * (K/64) * 16384 + 4 * s * M * (N + r)
 * bytes, s = K/256 when K is a multiple of 256 and 1 otherwise (room for a tiled weight, the
 * adapter rows and the fp32 split-K partial sums).  Larger problems return PBD_ERR_CAPACITY
 * before anything is launched, and the message gives both sizes; use pbd_op_linear for them.
 * Within 16 MiB fit, for instance, an N = 6144, K = 1024 weight with r = 16 up to M = 39, and
 * an N = 1024, K = 3072 weight with r = 16 up to M = 194.
 *
 * Zeroing: every call clears, on d_stream, the one part of the scratch that must start at zero,
 * the kernel's status word.  Every other byte a call reads there is written by that same call
 * first, so a call never sees an earlier call's data.
 *
 * Device errors: as for pbd_op_linear, the return value covers argument checks and launches;
 * pbd_op_linear_static_status reports a device wait that ran out.  Ask before the next call on
 * the device, which clears the status word.
 *
 * Concurrency: all calls on one device share the same scratch.  Two calls whose work can
 * overlap in time on the device (different streams without an ordering between them, or
 * several host threads with their own streams) race on it and can produce wrong results.
 * Issue them on one stream, or order the streams.
 *
 * Arguments as pbd_op_linear, without d_ws and ws_bytes; the work runs on the current device
 * and d_stream must belong to it.  Returns PBD_ERR_INVALID_ARG for unsupported sizes or null
 * pointers, PBD_ERR_CAPACITY when the scratch is too small, PBD_ERR_CUDA when a runtime call
 * fails (message from pbd_op_last_error()). */
pbd_status pbd_op_linear_static(int32_t M, int32_t K, int32_t N, int32_t r, float scale, const void *d_x,
                                const void *d_w, const void *d_a, const void *d_b, void *d_y, void *d_stream);

/* Device status of the last pbd_op_linear_static call on the current device: waits for d_stream,
 * then reads the status word in the library's static scratch.  PBD_OK (and *h_device_code = 0)
 * when no kernel latched an error; PBD_ERR_DEVICE with the latched code (the DEV_* values of the
 * pass kernel: 1 copy, 2 accumulation, 3 ring slot, 6 inputs) in *h_device_code otherwise, in
 * which case that call's y is invalid; PBD_ERR_STATE if no call was made on this device yet;
 * PBD_ERR_CUDA if the stream failed.  h_device_code may be NULL.  Allocates nothing. */
pbd_status pbd_op_linear_static_status(void *d_stream, int32_t *h_device_code);

/* Workspace bytes pbd_op_lm_head_argmax needs (0 if unsupported). */
size_t pbd_op_lm_head_workspace_bytes(int32_t M, int32_t H, int32_t V);

/* Tied lm_head with greedy readout (Section 3, step 4 uses the verifier's top-1 token):
 *     logits = x E^T (fp32, never rounded),  ids[m] = argmax_v logits[m, v], lowest v on ties.
 * d_x [M, H] and d_embed [V, H] bf16 row-major; d_ids [M] int32; d_logits_opt [M, V] fp32 or
 * NULL.  Requirements: V % 128 == 0, H % 64 == 0, 1 <= M <= 256.  The workspace's first word is
 * the kernel's status word: pbd_op_status(d_ws, ...) reports a device wait that ran out.  Its size
 * counts a copy of d_embed, which is made only where d_logits_opt lies over d_embed. */
pbd_status pbd_op_lm_head_argmax(int32_t M, int32_t H, int32_t V, const void *d_x, const void *d_embed,
                                 int32_t *d_ids, float *d_logits_opt, void *d_ws, size_t ws_bytes, void *d_stream);

/* Types of values that the calls below take. */
typedef enum { PBD_BF16 = 0, PBD_FP16 = 1, PBD_FP32 = 2 } pbd_dtype;

/* A paged key-value cache that the caller owns: one layer's K and V for `batch` sequences.
 * Slot j of sequence b is slot j % page_size of page d_page_table[b * max_pages + j / page_size]; its K (and likewise V)
 * of one head starts at d_k + page * stride_page + head * stride_head + (j % page_size) * stride_slot, strides in
 * values, head_dim values in a row.  [page][head][slot][d] and [page][slot][head][d] are both expressed so.
 * Requirements: head_dim 64, 128 or 256; d_k and d_v 16-byte aligned and every stride a multiple of 8; batch <= 1024;
 * no stride times its number of pages, heads or slots (in all calls: of rows) beyond 2^60 values.
 * Calls that write rows (a new token's, eviction's moves): each stride is at least what the dimensions of smaller strides span,
 * and no row of K lies over one of V; they may lie in turns in one buffer.
 * Pages of a sequence's slots [0, d_lens[b]) are read; table entries behind them are not.  Sequences may share pages that
 * a call only reads, and strides may then be 0.  Which token a slot holds is up to the caller: attention does not depend on the order. */
typedef struct {
    void *d_k, *d_v;
    int32_t dtype;                    /* PBD_BF16 or PBD_FP16 */
    int32_t n_pages, page_size, n_kv_heads, head_dim, batch, max_pages;
    int64_t stride_page, stride_head, stride_slot;
    const int32_t *d_page_table;      /* [batch, max_pages] */
    const int32_t *d_lens;            /* [batch] cached tokens, 0 to max_pages * page_size */
    float *d_weights;                 /* [batch, n_kv_heads, max_pages * page_size] accumulated attention weight, or NULL */
    int32_t *d_positions;             /* the same shape: position of the token in each slot, or NULL */
} pbd_kv_pages;

/* Workspace bytes pbd_op_decode_attention needs (0 if unsupported); only the cache's sizes, strides and type are read.  With
 * accumulate it has a score for every query head and slot of the tables, 4 * batch * n_q_heads * max_pages * page_size bytes of it. */
size_t pbd_op_decode_attention_workspace_bytes(const pbd_kv_pages *kv, int32_t n_q_heads, int32_t accumulate);

/* Attention of one new token per sequence over a paged cache (the attention step of a plain decoding pass, on the
 * caller's own cache): query head h reads KV head h / (n_q_heads / n_kv_heads),
 *     s_j = q . k_j,  p = softmax(scale * s),  out = sum_j p_j v_j,  lse = ln sum_j exp(scale * s_j).
 * d_q: batch rows q_stride values apart of [n_q_heads, head_dim]; d_out [batch, n_q_heads, head_dim]; both of the cache's
 * type.  d_lse_opt [batch, n_q_heads] fp32 or NULL.  A sequence without a slot gets zeros and -inf.
 * d_k_new, d_v_new (both or neither): the new token's own K and V, batch rows new_stride values apart of [n_kv_heads,
 * head_dim].  They are stored into slot d_lens[b] (whose page the table must name) and attended to as well; its position
 * goes to d_positions from d_new_positions [batch] when both are there.  d_lens is not changed: a layer's call leaves it
 * to the caller, who raises it once all layers are through.
 * accumulate: adds to d_weights[b, kv head, j] the p_j of all query heads of the group; the slot of a new token starts
 * from 0.  The sums run in an order fixed by the sizes and lengths: repeated calls give the same bits.
 * Score, softmax and output sums are fp32; p is split into two 16-bit parts for the tensor cores, so that the output's
 * error is that of its one rounding.
 * Attended values of V are finite, in bf16 at most 2^123 / slots (fp32 sums of p v, p up to 16, must not overflow): an infinite one
 * makes its dimension of the head's outputs NaN or infinite, and no other.
 * Requirements: n_q_heads a multiple of n_kv_heads; scale > 0; d_q, d_out, d_k_new and d_v_new 16-byte aligned, row strides
 * multiples of 8; nothing that the call writes (d_out, d_lse_opt, the workspace; with a new token K, V and positions; with accumulate
 * the weights) lies over anything else that it reads or writes.  The workspace (1024-byte aligned) is scratch; its first word
 * is the status word for pbd_op_status: a length outside [0, max_pages * page_size] (with a new token: one less) or a
 * page outside [0, n_pages) is reported there.  The call then means nothing for that sequence, but does no harm: one with such
 * a length counts as empty, and slots of such a page, a new token's too, are left out: they take no part in the softmax,
 * and their K, V, weights and positions stay as they are (in a KV head one of whose scores is NaN all weights become NaN). */
pbd_status pbd_op_decode_attention(const pbd_kv_pages *kv, int32_t n_q_heads, float scale, const void *d_q, int64_t q_stride,
                                   const void *d_k_new, const void *d_v_new, int64_t new_stride,
                                   const int32_t *d_new_positions, int32_t accumulate, void *d_out, float *d_lse_opt,
                                   void *d_ws, size_t ws_bytes, void *d_stream);

/* Workspace bytes pbd_op_evict needs (0 if unsupported); only the cache's sizes, strides and type are read. */
size_t pbd_op_evict_workspace_bytes(const pbd_kv_pages *kv, int32_t n_keep);

/* Eviction from a paged cache by accumulated attention weight.  Of the d_lens[b] slots of each sequence and KV head the
 * min(d_lens[b], n_keep) that rank first stay: slots whose position is below n_sink or at least d_next_positions[b] -
 * n_recent, then by d_weights (NaN last), equal ones by the lower slot.  Kept slots at or behind n_keep move (K, V, weight,
 * position) into the places in front that came free, the i-th into the i-th; all others stay where they are, so the
 * kept ones are slots [0, n_keep) afterwards, in no order of their tokens.  Sequences of at most n_keep slots keep all.
 * K and V move in place.  Weights and positions of the kept slots go to d_out_weights and d_out_positions, shaped like
 * d_weights and d_positions: those arrays themselves, or others apart from them and from one another; slots behind the kept ones are not
 * written.  d_lens is not changed: the caller lowers it to at most n_keep once all layers are through.
 * Requirements: n_recent + n_sink <= n_keep; no page in use is named twice, by one sequence or two; nothing that the call writes (K, V, the outputs, the
 * workspace) lies over anything else that it reads or writes, weights and positions as their own outputs apart.  The workspace (1024-byte aligned) is scratch;
 * its first word is the status word for pbd_op_status: a length outside [0, max_pages * page_size], whose sequence is left as it
 * is, or a page outside [0, n_pages) among those of a sequence that evicts.  A move from or to a slot of such a page is left
 * out whole: row, weight and position. */
pbd_status pbd_op_evict(const pbd_kv_pages *kv, int32_t n_keep, int32_t n_recent, int32_t n_sink,
                        const int32_t *d_next_positions, float *d_out_weights, int32_t *d_out_positions, void *d_ws,
                        size_t ws_bytes, void *d_stream);

/* Workspace bytes pbd_op_token_logprobs needs (0 if unsupported). */
size_t pbd_op_token_logprobs_workspace_bytes(int32_t M, int32_t V, int32_t k);

/* Log probabilities of given tokens, entropy and top alternatives of M rows of V logits (those of pbd_op_lm_head_argmax,
 * pbd_verify_block or pbd_decode_step, or the caller's), in one pass over them:
 *     p = softmax(x / temperature),  logprob = ln p[token],  entropy = -sum p ln p,
 *     top_ids / top_logprobs: the k likeliest, by logit, equal ones by the lower id.
 * d_logits: rows ld values apart, of type dtype (pbd_dtype).  d_tokens_opt [M] with d_logprob_opt [M] fp32, both or
 * neither: a negative token asks for nothing (its log probability is 0), one at or above V is reported by
 * pbd_op_status (DEV_BAD_TOKEN) and gives NaN.  d_entropy_opt [M] fp32 or NULL.  d_top_ids [M, k] int32 and
 * d_top_logprobs [M, k] fp32, not read for k = 0.  Logits of -inf are masked; a row with nothing else has log
 * probabilities of -inf and entropy 0.  A row that holds NaN or +inf gives NaN (and ids that say nothing).
 * Requirements: 1 <= M <= 2^30, 1 <= V <= 2^30, ld >= V, 0 <= k <= min(32, V); temperature > 0; no output lies over the logits, the
 * tokens, the workspace or another output.  Sums are fp32.  The workspace (1024-byte aligned) is scratch; its first word is
 * the status word for pbd_op_status. */
pbd_status pbd_op_token_logprobs(int32_t M, int32_t V, int32_t dtype, const void *d_logits, int64_t ld, float temperature,
                                 const int32_t *d_tokens_opt, int32_t k, float *d_logprob_opt, float *d_entropy_opt,
                                 int32_t *d_top_ids, float *d_top_logprobs, void *d_ws, size_t ws_bytes, void *d_stream);

/* Workspace bytes pbd_op_assign_pages needs (0 if unsupported). */
size_t pbd_op_assign_pages_workspace_bytes(int32_t batch);

/* Pages for the next tokens of every sequence, and the packed rows' slots, from lengths in device memory: what a step does
 * before its layers.  Sequence b has d_lens[b] cached tokens and gets d_n_new[b] more; afterwards it holds exactly the
 * ceil((d_lens[b] + d_n_new[b]) / page_size) pages at the front of its table row, so that a sequence that has ended
 * (both 0) gives all of its pages back, and one that was cut back those behind its end.
 * Held pages: d_held[b] entries of d_page_table [batch, max_pages].  Free ones: a stack, d_free [n_pages], of *d_n_free
 * entries, the last on top.  First the sequences give back, in their order and each its entries in theirs, then they take from the top,
 * in the same order.  Entries of a table row behind those held, and of d_free at or behind the new *d_n_free, stay as they were.
 * Outputs: d_starts [batch + 1], the packed rows of sequence b being [d_starts[b], d_starts[b + 1]); for each packed row its
 * slot page * page_size + place in the page in d_slots [max_new], and its position d_lens[b] + i in d_positions_opt
 * [max_new] or NULL.  Rows behind the last sequence's get -1 and 0: max_new may be a captured step's largest size.
 * d_lens is not changed: the caller raises it once all layers are through.
 * The workspace (1024-byte aligned) is scratch; its first word is the status word for pbd_op_status: 5 a length below 0 or
 * beyond max_pages * page_size, or more than max_new new tokens; 7 a page outside [0, n_pages) among those given or taken, or held and
 * free ones of more than n_pages in all; 8 not enough free pages.  Nothing is assigned then: table, held and free pages
 * stay as they were, the starts are 0 and all slots -1.  (7 with starts: a page held before lies outside; its rows' slots are -1.)
 * Requirements: batch <= 1024; max_pages * page_size <= 2^30; max_new <= 2^30; no page is held or free twice; nothing that the call
 * writes lies over anything else that it reads or writes. */
pbd_status pbd_op_assign_pages(int32_t batch, int32_t max_pages, int32_t page_size, int32_t n_pages, const int32_t *d_lens,
                               const int32_t *d_n_new, int32_t *d_page_table, int32_t *d_held, int32_t *d_free,
                               int32_t *d_n_free, int32_t max_new, int32_t *d_starts, int64_t *d_slots,
                               int32_t *d_positions_opt, void *d_ws, size_t ws_bytes, void *d_stream);

/* Workspace bytes pbd_op_prompt_attention needs (0 if unsupported). */
size_t pbd_op_prompt_attention_workspace_bytes(int32_t T, int32_t batch, int32_t n_q_heads, int32_t n_kv_heads,
                                               int32_t head_dim);

/* Attention over whole prompts, causal: T packed rows of `batch` sequences, sequence b the rows [d_starts[b], d_starts[b + 1]);
 * row i of a sequence sees its rows 0 to i.  Query head h reads KV head h / (n_q_heads / n_kv_heads),
 *     s_j = q . k_j,  p = softmax(scale * s),  out = sum_j p_j v_j,  lse = ln sum_j exp(scale * s_j).
 * d_q: T rows q_stride values apart of [n_q_heads, head_dim]; d_k, d_v: T rows kv_stride values apart of [n_kv_heads, head_dim], so that the
 * three may be parts of one projection's rows; d_out [T, n_q_heads, head_dim]; all of type dtype, PBD_BF16 or PBD_FP16.
 * d_lse_opt [T, n_q_heads] fp32 or NULL.  Rows of no sequence are neither read nor written.  A row sees rows of the call alone, nothing that
 * is cached already: prompts begin at an empty cache, or come whole.
 * kv_opt with d_slots_opt [T] (both or neither): K and V of each sequence's row t are stored into slot d_slots_opt[t] of the cache (its page's
 * number times page_size plus the place there, as pbd_op_assign_pages gives it); negative: not stored.  Of the cache K, V, sizes and strides
 * count, not table and lengths (which have to be named all the same).
 * Score, softmax and output sums are fp32; p is rounded to the type for the tensor cores (relative to the row's largest weight, so the
 * error is a rounding's share of each p_j v_j), and out once more.
 * A value of V that is infinite or NaN makes its dimension NaN or infinite in the outputs of the rows and heads that see it, and
 * no other; K and V of rows that a row does not see do not touch it, whatever they hold.  Finite values of V: in bf16 at most 2^123 / T
 * (fp32 sums of p v, p up to 16, must not overflow).
 * Requirements: head_dim 64, 128 or 256; n_q_heads a multiple of n_kv_heads; batch <= 1024; scale > 0; d_q, d_k, d_v and d_out 16-byte
 * aligned, row strides multiples of 8 below 2^38; no slot twice; nothing that the call writes lies over anything else that it reads or writes.
 * The workspace (1024-byte aligned) is scratch; its first word is the status word for pbd_op_status: 5 a sequence whose bounds
 * descend or lie outside [0, T], or that begins below any bound in front of its own: its rows are left out (so no row is two sequences');
 * 7 a slot outside the cache, whose row is not stored. */
pbd_status pbd_op_prompt_attention(int32_t T, int32_t batch, int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim,
                                   int32_t dtype, float scale, const void *d_q, int64_t q_stride, const void *d_k,
                                   const void *d_v, int64_t kv_stride, const int32_t *d_starts, const pbd_kv_pages *kv_opt,
                                   const int64_t *d_slots_opt, void *d_out, float *d_lse_opt, void *d_ws, size_t ws_bytes,
                                   void *d_stream);

/* Workspace bytes pbd_op_tree_attention needs (0 if unsupported); only the cache's sizes, strides and type are read. */
size_t pbd_op_tree_attention_workspace_bytes(const pbd_kv_pages *kv, int32_t T, int32_t n_q_heads);

/* Attention of up to 64 drafted tokens a sequence over a paged cache (the attention step of a verify pass, on the caller's own
 * cache): T packed rows, sequence b the rows [d_starts[b], d_starts[b + 1]), its nodes in order.  d_parents_opt [T]: the node of the
 * same sequence that a node follows, before it, or -1 for one that follows the cached tokens; NULL: each node follows the one before it (a
 * verify block).  Node i sees the d_lens[b] cached slots, its ancestors and itself; formulas, heads, d_q and d_out as
 * pbd_op_prompt_attention.  A row that sees nothing gets zeros and -inf.
 * d_k_new, d_v_new: the nodes' own K and V, T rows new_stride values apart of [n_kv_heads, head_dim].  They are stored into slots
 * d_lens[b] + i (whose pages the table must name), and node i's position goes to d_positions from d_new_positions_opt [T]
 * when both are there.  d_lens and d_weights are not changed.  pbd_op_commit_path then makes an accepted path contiguous.
 * Rounding, infinite and NaN values of V as pbd_op_prompt_attention; a node does not touch those that do not descend from it.  Finite values of
 * V, cached ones and nodes' own: in bf16 at most 2^123 / (d_lens[b] + nodes), the keys that a row's sums may have (not / T).
 * Requirements: T <= 2^30; scale > 0; d_q, d_k_new, d_v_new and d_out 16-byte aligned, row strides multiples of 8 below 2^38; no page
 * in use is named twice among those that new rows go to; nothing that the call writes lies over anything else that it reads or writes; the
 * table has room for no more than 2^31 - 2 places in all (else PBD_ERR_CAPACITY, and 0 workspace bytes): with R = min(64, T) *
 * (n_q_heads / n_kv_heads), each of min(batch, T) sequences, n_kv_heads heads and ceil(R / 256) chunks (head_dim 256: ceil(R / 128)) counts 4
 * places and one for every 128 slots of its table row; at head_dim 64 10 and two, three where R > 128.
 * The workspace (1024-byte aligned) is scratch; its first word is the status word for pbd_op_status: 5 bounds that descend, lie outside [0, T]
 * or span more than 64 rows, a sequence that begins below any bound in front of its own, or a length outside [0, max_pages * page_size -
 * nodes]: the sequence is left out; 7 a page outside [0, n_pages): its slots, new nodes' among them, take no part and are not stored; 9 a
 * parent that is not before its node: it counts as -1. */
pbd_status pbd_op_tree_attention(const pbd_kv_pages *kv, int32_t T, int32_t n_q_heads, float scale, const void *d_q,
                                 int64_t q_stride, const void *d_k_new, const void *d_v_new, int64_t new_stride,
                                 const int32_t *d_starts, const int32_t *d_parents_opt, const int32_t *d_new_positions_opt,
                                 void *d_out, float *d_lse_opt, void *d_ws, size_t ws_bytes, void *d_stream);

/* Workspace bytes pbd_op_commit_path needs (0 if unsupported); only the cache's sizes, strides and type are read. */
size_t pbd_op_commit_path_workspace_bytes(const pbd_kv_pages *kv, int32_t max_path);

/* Makes the accepted path of each sequence's drafted tree contiguous behind its cached tokens: K, V and, where the cache has them,
 * weight and position of slot d_lens[b] + d_path[b * max_path + i] go to slot d_lens[b] + i, for i < d_n_accepted[b].  A path names nodes in
 * ascending order (a node comes after its parent), the first of them 0 or above; entries behind d_n_accepted[b] are not read.  Other slots stay
 * as they are.  d_lens is not changed: a layer's call leaves it to the caller, who adds the accepted numbers once all layers are through.
 * Requirements: 1 <= max_path <= 64; no page in use is named twice; nothing that the call writes (K, V, weights, positions, the workspace)
 * lies over anything else that it reads or writes.  The workspace (1024-byte aligned) is scratch; its first word is the status word for
 * pbd_op_status: 5 a number outside [0, max_path] or a length outside [0, max_pages * page_size], 9 a path that does not
 * ascend or leaves the tree's 64 nodes or the table: that sequence is left as it is, whatever its pages are; 7 a page outside
 * [0, n_pages): moves from and to its slots are left out.  (Of several sequences' faults one is reported.) */
pbd_status pbd_op_commit_path(const pbd_kv_pages *kv, const int32_t *d_path, int32_t max_path, const int32_t *d_n_accepted,
                              void *d_ws, size_t ws_bytes, void *d_stream);

/* Device status of the last call of an entry point above that used the workspace d_ws (the 1024-byte-aligned
 * pointer that call was given): waits for d_stream, then reads the status word at the start of d_ws.  PBD_OK when no
 * kernel latched an error; PBD_ERR_DEVICE with the latched code in *h_device_code (may be NULL) otherwise, and that
 * call's outputs are invalid; PBD_ERR_INVALID_ARG for a null or misaligned d_ws; PBD_ERR_CUDA if the stream failed.
 * What kernels latch: a device wait that runs out, after one second (1, 2, 3 or 6: linear, lm_head, token_logprobs, prompt and tree
 * attention; in the last two one and 32 us for each 128 keys of a call's longest possible work between two waits), and lengths, pages (7;
 * 8: none left), trees (9) and tokens (4) in device memory that lie outside their range (5: a length), which the host cannot check. */
pbd_status pbd_op_status(const void *d_ws, void *d_stream, int32_t *h_device_code);

/* Message of the last failed pbd_op_* call on this thread ("" if none). */
const char *pbd_op_last_error(void);

#ifdef __cplusplus
}
#endif
#endif /* PBD_OPS_H */
