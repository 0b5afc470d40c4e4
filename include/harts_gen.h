/*
 * harts_gen -- sampling on rollout trees for sm_100a (B200): C ABI.
 *
 * (No counterpart in the paper, which trains on finished trees: these calls are the serving form of the same layers, for the
 * policy that writes the trees token by token.)
 *
 * Three things a decoding step of a hybrid model does:
 *   harts_gen_la            the recurrence of harts_la.h from and into kept states: one token, drafted tokens, turns, prompts
 *   harts_gen_cache_*       keys and values into a paged cache (bf16, or 8 bits with a scale for each token and head), and back
 *   harts_gen_attn          softmax attention of the sampled tokens on the cached tree (the visibility of harts_attn.h): a prefix
 *                           that branches share is read once for all of them
 *
 * Conventions are those of harts_la.h: int32 status returns, no allocation of device memory by the library, kernels enqueued on
 * the caller's stream (a cudaStream_t as void*, of the current device) without synchronising, no CPU fallback.  All pointers are
 * DEVICE pointers unless a comment says host; base pointers are 16-byte aligned.  Every call may be captured into a CUDA graph.
 * dev_status: int32[2] device or NULL; an index out of range is met by leaving out what it names, with dev_status[0] = HARTS_EINVAL and
 * dev_status[1] = its position (read with harts_la_check(); the caller zeroes the word).
 */
#ifndef HARTS_GEN_H_
#define HARTS_GEN_H_

#include <stddef.h>
#include <stdint.h>

#include "harts_la.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * Linear attention with a decay for each head, from and into kept states (Eq. 1 with a scalar gate, as in harts_la.h):
 *
 *     S_t = exp(g_t) S_{t-1} + k_t^T v_t,     o_t = q_t S_t
 *
 *   n_seq sequences; sequence i is rows [seq_begin[i], seq_begin[i] + seq_len[i]) of q, k, v, g, o, 0 <= seq_len[i] <= max_len.
 *   in_state[i]:  the state it starts from (an index into states), -1: zero
 *   out_state[i]: where its last state goes, -1: it is not kept.  May be in_state[i].  No two sequences have the same
 *                 out_state, and none has another one's out_state as its in_state (several may start from the same state, which is how
 *                 branches fork): what such a call leaves in the state, and reads from it, is undefined.
 *   seq_begin, seq_len, in_state, out_state: device int32 [n_seq] (a draft's accepted length can come straight from a kernel)
 *   max_len: host; a bound on the lengths.  It and n_rows choose the form: tokens one by one with the state in registers, or chunks
 *            of 64 on the tensor cores.
 *   q, k [n_rows, H, dk], v [n_rows, H, dv] in `dtype`, heads contiguous, ld_q, ld_k, ld_v elements between rows (>= H d, a multiple
 *            of 16 bytes); g fp32 [n_rows, H], <= 0 (minus infinity too: the state is forgotten); o [n_rows, H, dv] contiguous, or NULL: only the states are wanted, q may be NULL
 *            then too.  Rows of no sequence are neither read nor written.
 *            Sequences do not share rows, and o overlaps no input: what is written then is undefined.
 *   states fp32 [n_states, H, dk, dv]: the layout of the slots of harts_la.h, so that a training forward's slots can be the pool.
 *   workspace: harts_gen_la_workspace_bytes(), for chunked calls only (NULL where that is 0).  Calls that share it, also as parts of
 *            captured graphs, must not run at the same time.
 * Served: fp32 with dk = dv = 64 or 128, bf16 with dk = dv = 64 or 128; chunks on the tensor cores for bf16 with 128, the others
 * walk token by token whatever their length.  States are fp32 and so are all sums; on the tensor cores the weighted keys are three bf16 terms each, so
 * that states keep fp32's accuracy, while scores and the states that outputs are made of are rounded to bf16, as in harts_la.h.
 * There, an infinity or a NaN in a row's k or v can also reach the outputs (not the states) of the rows ahead of it in its chunk, and an infinity
 * in k makes NaN of what it makes infinite token by token.
 * A sequence with a bad entry is left out (dev_status[1] = its number).
 * Errors: HARTS_EINVAL (null or misaligned pointer, size out of range, workspace too small), HARTS_EUNSUPPORTED, HARTS_ECUDA.
 */
int32_t harts_gen_la_workspace_bytes(int32_t n_seq, int32_t max_len, int64_t n_rows, int32_t H, int32_t dk, int32_t dv,
                                     int32_t dtype, size_t* bytes);
int32_t harts_gen_la(int32_t n_seq, const int32_t* seq_begin, const int32_t* seq_len, const int32_t* in_state,
                     const int32_t* out_state, int32_t max_len, int64_t n_rows, const void* q, int64_t ld_q, const void* k,
                     int64_t ld_k, const void* v, int64_t ld_v, const float* g, void* o, float* states, int32_t n_states, int32_t H,
                     int32_t dk, int32_t dv, int32_t dtype, void* workspace, size_t workspace_bytes, int32_t* dev_status,
                     void* stream);

/*
 * Paged cache of keys and values, d = 128.
 *   k_cache, v_cache [n_pages, Hkv, page, 128]: a token's row lies in slot = page number * page + place in the page; page is 16, 32,
 *   64 or 128, n_pages * page and n_pages * Hkv at most INT32_MAX
 *   cache_type HARTS_BF16: the rows as they are; k_exp, v_exp NULL
 *   cache_type HARTS_E4M3: 8-bit values y with a power of two for each (token, head): row = y 2^(exp - 127), exp in k_exp, v_exp
 *              uint8 [n_pages, Hkv, page].  The power is the smallest with max |row| <= 448 2^e (not below 2^-126), so that y is the row's
 *              values rounded to 4 significant bits, to nearest even, whatever their size, and reading back is exact (what would round to
 *              2^128 becomes the value below it).  A row with an infinity
 *              or a NaN becomes all NaN: exp 255, values zero.
 *
 * harts_gen_cache_write: rows of k, v (bf16 [n, Hkv, 128], heads contiguous, ld_k, ld_v elements between rows) into slots slot[i]
 * (device int32 [n]); slot[i] < 0: the row is left out (a padded batch).  Two rows of a call have different slots (or what stays
 * is undefined).  A slot beyond the cache is left out and reported.
 * harts_gen_cache_read: the rows of slots slot[i] into k, v (bf16 [n, Hkv, 128], contiguous); slot[i] < 0 and slots beyond the cache
 * (reported) give zeros.  Either of k, v may be NULL.
 */
#define HARTS_E4M3 2
int32_t harts_gen_cache_write(int64_t n, const int32_t* slot, const void* k, int64_t ld_k, const void* v, int64_t ld_v, void* k_cache,
                              void* v_cache, uint8_t* k_exp, uint8_t* v_exp, int32_t n_pages, int32_t page, int32_t Hkv, int32_t d,
                              int32_t cache_type, int32_t* dev_status, void* stream);
int32_t harts_gen_cache_read(int64_t n, const int32_t* slot, const void* k_cache, const void* v_cache, const uint8_t* k_exp,
                             const uint8_t* v_exp, void* k, void* v, int32_t n_pages, int32_t page, int32_t Hkv, int32_t d,
                             int32_t cache_type, int32_t* dev_status, void* stream);

/*
 * Attention of sampled tokens on the cached tree.  The cached forest is given like a training forest (tree_node_ptr, node_parent,
 * node_fork_off, node_len as for harts_la_plan(), but node_len may be 0 and a fork offset anything from 0 to its parent's length); node
 * v's token j is in slot node_page[node_page_ptr[v] + j / page] * page + j % page of the cache.  Query r belongs to node q_node[r] and
 * sees that node's tokens 0 .. q_pos[r] and, of every ancestor, the tokens ahead of the fork:
 *
 *     o_r = sum_j softmax_j(scale q_r . k_j) v_j,     lse_r = log sum_j exp(scale q_r . k_j)     (per query head; kv head = head / (Hq / Hkv))
 *
 * A branch that decodes one token has one query (its newest token, whose key is in the cache already); drafted tokens are more queries
 * of the same node.  q_node[r] < 0, and a query that sees nothing: o = 0, lse = -inf.  Stored tokens that a query does not see may hold anything,
 * infinities and NaN too.
 *
 * harts_gen_attn_index (host in, host out): work lists for such a forest, one int32 blob; the same blob is copied to the device.
 *   Tokens that several queries see are read once for up to 128 rows (a row: a query and a head of its group), long runs are split over the GPU.
 *   grow: by how many tokens nodes with queries may grow while the index is used: between calls (and replays of a captured call) q_pos may
 *   go up, to node_len - 1 + grow at most and as far as the node's listed pages go, and never below what it was for the index.
 *   A new branch, a fork, or a query more or less needs a new index.  Work is divided as if all that room were tokens, so ask for what will be
 *   used: 64 branches of 1,200 on 16,421 tokens take 64 us with no room, 66 with 256 tokens of it, 88 with 1,024, 100 with 4,096.
 *   cap_words: capacity of blob, which may be NULL to get *n_words only.
 *   Errors: HARTS_EINVAL (malformed forest, pages missing or negative, q_pos out of range, capacity), HARTS_ENOMEM.
 * harts_gen_attn_workspace_bytes: of the parts of split sums.  Calls that share a workspace must not run at the same time.
 * harts_gen_attn: q bf16 [n_q, Hq, 128], heads contiguous, ld_q elements between rows; q_pos device int32 [n_q]; o bf16, lse fp32,
 *   contiguous, written for every query, neither overlapping an input.  An out-of-range q_pos is brought into its range and reported (dev_status[1] = the query).
 *   scale is positive and at most FLT_MAX ln 2 (2.3e38).  Products on the tensor cores with fp32 sums; softmax in fp32, its values rounded for the
 *   second product: to bf16, or, of an 8-bit cache, to fp16 in the kernel for up to 16 rows.
 */
#define HARTS_GEN_ATTN_HEADER_WORDS 32
int32_t harts_gen_attn_index(int32_t n_trees, const int32_t* tree_node_ptr, const int32_t* node_parent, const int32_t* node_fork_off,
                             const int32_t* node_len, const int32_t* node_page_ptr, const int32_t* node_page, int32_t page, int32_t n_q,
                             const int32_t* q_node, const int32_t* q_pos, int32_t Hq, int32_t Hkv, int32_t grow, int64_t cap_words,
                             int32_t* blob, int64_t* n_words);
int32_t harts_gen_attn_workspace_bytes(const int32_t* host_index, size_t* bytes);
int32_t harts_gen_attn(const int32_t* host_index, const int32_t* dev_index, const void* q, int64_t ld_q, const void* k_cache,
                       const void* v_cache, const uint8_t* k_exp, const uint8_t* v_exp, int32_t n_pages, int32_t cache_type,
                       const int32_t* q_pos, void* o, float* lse, float scale, void* workspace, size_t workspace_bytes,
                       int32_t* dev_status, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* HARTS_GEN_H_ */
