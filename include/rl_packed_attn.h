/*
 * rl_packed_attn -- causal attention over packed sequences with grouped heads, and its gradient, for AMD MI355X
 * (gfx950).  C ABI.
 *
 * The policy update (Sec. 3.2.2 "Policy update stage") runs the policy over whole trajectories, whose lengths differ: their
 * tokens lie one sequence after the other in one row of tokens, without padding.  rl_prefill_attn is the rollout's pass over
 * prompts, in the padded layout of the decode stores and without a gradient.  For query head h, j = h / (Hq / Hkv), token i of
 * sequence s, i.e. cu_seqlens[s] <= i < cu_seqlens[s + 1]:
 *
 *   z_n       = scale * <q[i,h], k[n,j]>                            cu_seqlens[s] <= n <= i
 *   lse[h,i]  = ln sum_n exp(z_n),     out[i,h] = sum_n exp(z_n - lse[h,i]) v[n,j]
 *
 * and from dout, with p_n = exp(z_n - lse[h,i]) and D[i,h] = sum_c dout[i,h,c] out[i,h,c]:
 *
 *   g_n       = p_n (<dout[i,h], v[n,j]> - D[i,h])
 *   dq[i,h]   = scale * sum_n g_n k[n,j]
 *   dk[n,j]   = scale * sum over i and the heads of j of g_n q[i,h]
 *   dv[n,j]   = sum over i and the heads of j of p_n dout[i,h]
 *
 * Tokens before cu_seqlens[0] or from cu_seqlens[n_seqs] on belong to no sequence: out 0, lse -inf, gradients 0.  Sequences
 * may be empty.  A key outside a row's range has no effect on the row, whatever it holds (infinities and NaN included).
 *
 * bf16 data, fp32 sums on the matrix cores; p and g are rounded to bf16 before their products (half a step of each term; backward,
 * rows of up to 64 keys and keys of up to 64 rows also take what that left over), results
 * once more.  Sums have a fixed order: results are bit-reproducible from call to call.
 */
#ifndef RL_PACKED_ATTN_H
#define RL_PACKED_ATTN_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

/* All pointers are DEVICE memory, borrowed until the enqueued work has run.  The heads of a token are contiguous, tokens a
 * stride (elements) apart.  bf16 tensors are 16-byte aligned, strides multiples of 8. */
typedef struct {
  uint32_t struct_size;      /* = sizeof(rl_packed_attn_desc)                                     */
  int32_t  dtype;            /* 1 (bf16); nothing else                                            */
  int64_t  T;                /* tokens (>= 0)                                                     */
  int32_t  n_seqs;           /* sequences (>= 0)                                                  */
  int32_t  Hq, Hkv, d;       /* Hq % Hkv == 0, Hq / Hkv <= 64, d = 64 or 128                      */
  float    scale;            /* |scale| <= 2e38                                                   */
  const void*    q;          /* [T, Hq, d]                                                        */
  const void*    k;          /* [T, Hkv, d]                                                       */
  const void*    v;          /* [T, Hkv, d]                                                       */
  const int32_t* cu_seqlens; /* [n_seqs + 1], not decreasing; read on the device                  */
  void*          out;        /* [T, Hq, d] bf16                                                   */
  float*         lse;        /* [Hq, T]; may be NULL                                              */
  int64_t q_stride, k_stride, v_stride, out_stride;
} rl_packed_attn_desc;

typedef struct {
  uint32_t struct_size;      /* = sizeof(rl_packed_attn_backward_desc)                            */
  int32_t  dtype;
  int64_t  T;
  int32_t  n_seqs;
  int32_t  Hq, Hkv, d;
  float    scale;
  const void*    dout;       /* [T, Hq, d]                                                        */
  const void*    q;          /* the forward call's inputs ...                                     */
  const void*    k;
  const void*    v;
  const void*    out;        /* ... and outputs                                                   */
  const float*   lse;
  const int32_t* cu_seqlens;
  void*          dq;         /* [T, Hq, d]  bf16                                                  */
  void*          dk;         /* [T, Hkv, d] bf16                                                  */
  void*          dv;         /* [T, Hkv, d] bf16                                                  */
  int64_t dout_stride, q_stride, k_stride, v_stride, out_stride, dq_stride, dk_stride, dv_stride;
  void*          workspace;  /* device scratch, 256-byte aligned, >= the query's bytes; one call's at a time */
  size_t         workspace_bytes;
} rl_packed_attn_backward_desc;

/*
 * Both: enqueue on `hip_stream` (hipStream_t as void*; NULL = default stream), asynchronous, allocate nothing.  Return 0
 * or a negative code with the meaning of the RLDA_ERR_* values of rl_decode_attn.h: -1 invalid argument (NULL where a tensor
 * is required, negative sizes, |scale| > 2e38 or NaN), -2 unsupported (dtype, d, head counts, strides or alignment, T > 2^24,
 * heads times tokens beyond a launch's 2^32 threads: T * Hq or T * Hkv from 2^29 on),
 * -3 workspace, -4 struct_size, -5 HIP error.  With T = 0 nothing is read or written.
 */
int rl_packed_attn(const rl_packed_attn_desc* desc, void* hip_stream);
int rl_packed_attn_backward(const rl_packed_attn_backward_desc* desc, void* hip_stream);

/* Bytes of workspace the backward call needs (0 if none or if the descriptor is invalid).  Pure host code. */
size_t rl_packed_attn_backward_workspace_bytes(const rl_packed_attn_backward_desc* desc);

#ifdef __cplusplus
}
#endif
#endif
