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
 *            of 16 bytes); g fp32 [n_rows, H], <= 0; o [n_rows, H, dv] contiguous, or NULL: only the states are wanted, q may be NULL
 *            then too.  Rows of no sequence are neither read nor written.
 *   states fp32 [n_states, H, dk, dv]: the layout of the slots of harts_la.h, so that a training forward's slots can be the pool.
 *   workspace: harts_gen_la_workspace_bytes(), for chunked calls only (NULL where that is 0).  Calls that share it, also as parts of
 *            captured graphs, must not run at the same time.
 * Served: fp32 with dk = dv = 64 or 128, bf16 with dk = dv = 64 or 128; chunks on the tensor cores for bf16 with 128, the others
 * walk token by token whatever their length.  States are fp32 and so are all sums; on the tensor cores the weighted keys are two bf16 terms each, so
 * that states keep fp32's accuracy, while scores and the states that outputs are made of are rounded to bf16, as in harts_la.h.
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

#ifdef __cplusplus
}
#endif
#endif /* HARTS_GEN_H_ */
