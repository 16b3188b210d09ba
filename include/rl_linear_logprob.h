/*
 * rl_linear_logprob -- per-token policy statistics straight from hidden states and the head's weights, and their
 * gradient, for AMD MI355X (gfx950).  C ABI.
 *
 * rl_token_logprob reads logits that somebody has kept.  Over a vocabulary of 150 thousand these are the largest tensor of
 * the policy update; here the product of hidden states and weights is made a piece of the vocabulary at a time and used up
 * where it is made, in both directions.  With z = inv_temperature * hidden . weight^T (one row per token), y_n = token_ids[n]:
 *
 *   lse[n]     = ln sum_v exp(z[n,v])
 *   logprob[n] = z[n, y_n] - lse[n]
 *   entropy[n] = - sum_v p_v ln p_v,                       p_v = exp(z[n,v] - lse[n])
 *
 * and from g_logprob[n] = d loss / d logprob[n] (what rl_policy_loss leaves) and g_entropy[n] = d loss / d entropy[n]:
 *
 *   dz[n,v]  = inv_temperature * (g_logprob[n] (1[v = y_n] - p_v) - g_entropy[n] p_v (ln p_v + entropy[n]))
 *   dhidden  = dz . weight,    dweight = dz^T . hidden
 *
 * Ids, masked logits and rows without a live logit are as in rl_token_logprob.h (a negative id: logprob 0; id >= vocab: NaN; a
 * logit of -inf or NaN is masked).  Backward, a masked logit has dz 0 and no part in dhidden, whatever its weights hold (it has both only where
 * its token was sampled); an id outside [0, vocab) has no gradient of its logprob; a row without any
 * gradient (both 0, or no live logit) adds nothing to dweight, whatever its hidden state holds, and gets dhidden 0.
 *
 * bf16 data on the matrix cores with fp32 sums; logits, statistics and p are fp32, dz is rounded to bf16 before its two
 * products (half a step of each term, as the results' own rounding; up to 32 rows also what that left over), gradients are rounded once.  All sums have a fixed
 * order: results are bit-reproducible from call to call.
 */
#ifndef RL_LINEAR_LOGPROB_H
#define RL_LINEAR_LOGPROB_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

/* All pointers are DEVICE memory, borrowed until the enqueued work has run.  bf16 tensors are 16-byte aligned, strides
 * (elements between rows) multiples of 8. */
typedef struct {
  uint32_t struct_size;      /* = sizeof(rl_linear_logprob_desc)                                  */
  int32_t  dtype;            /* of hidden and weight: 1 (bf16); nothing else                      */
  int64_t  n_rows;           /* tokens (>= 0)                                                     */
  int32_t  vocab, hidden;    /* weight rows (>= 1); columns (a multiple of 8, >= 8)               */
  float    inv_temperature;  /* positive, finite                                                  */
  const void*    hidden_states;  /* [n_rows, hidden], hidden_stride                               */
  const void*    weight;         /* [vocab, hidden],  weight_stride                               */
  const int32_t* token_ids;      /* [n_rows]                                                      */
  float* logprob;            /* [n_rows] each; any may be NULL                                    */
  float* lse;
  float* entropy;
  int64_t hidden_stride, weight_stride;
  void*  workspace;          /* device scratch, 256-byte aligned, >= the query's bytes; one call's at a time */
  size_t workspace_bytes;
} rl_linear_logprob_desc;

typedef struct {
  uint32_t struct_size;      /* = sizeof(rl_linear_logprob_backward_desc)                         */
  int32_t  dtype;
  int64_t  n_rows;
  int32_t  vocab, hidden;
  float    inv_temperature;
  const void*    hidden_states;
  const void*    weight;
  const int32_t* token_ids;
  const float*   lse;        /* [n_rows] from the forward call                                    */
  const float*   entropy;    /* [n_rows] from the forward call; needed with g_entropy             */
  const float*   g_logprob;  /* [n_rows]                                                          */
  const float*   g_entropy;  /* [n_rows] or NULL                                                  */
  void*  dhidden;            /* [n_rows, hidden] bf16, dhidden_stride, or NULL (not computed)     */
  void*  dweight;            /* [vocab, hidden] bf16, dweight_stride, written (not added to), or NULL */
  int64_t hidden_stride, weight_stride, dhidden_stride, dweight_stride;
  void*  workspace;          /* as above                                                          */
  size_t workspace_bytes;
} rl_linear_logprob_backward_desc;

/*
 * Both: enqueue on `hip_stream` (hipStream_t as void*; NULL = default stream), asynchronous, allocate nothing.  Return 0
 * or a negative code with the meaning of the RLDA_ERR_* values of rl_decode_attn.h: -1 invalid argument (NULL where a tensor
 * is required, sizes below their least, inv_temperature), -2 unsupported (dtype, hidden not a multiple of 8, strides or
 * alignment, n_rows or vocab > 2^24, n_rows * vocab > 2^45, hidden or strides > 2^20), -3 workspace, -4 struct_size, -5 HIP error.
 * With n_rows = 0 nothing is read and dweight is set to zeros.
 */
int rl_linear_logprob(const rl_linear_logprob_desc* desc, void* hip_stream);
int rl_linear_logprob_backward(const rl_linear_logprob_backward_desc* desc, void* hip_stream);

/* Bytes of workspace the calls need (0 if none or if the descriptor is invalid).  Pure host code; looks at n_rows, vocab, hidden
 * and, backward, at which of dhidden and dweight are NULL. */
size_t rl_linear_logprob_workspace_bytes(const rl_linear_logprob_desc* desc);
size_t rl_linear_logprob_backward_workspace_bytes(const rl_linear_logprob_backward_desc* desc);

#ifdef __cplusplus
}
#endif
#endif
