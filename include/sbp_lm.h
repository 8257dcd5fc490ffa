/*
 * sbp_lm.h -- C ABI of the steps a language model's block has between its linear layers, and of the token table below
 * the first block, under Stochastic Backpropagation (SBP) on AMD MI355X (gfx950).  Same library, conventions, element
 * types, flags and status codes as sbp.h: device pointers, dense row-major tensors, nothing allocated, arguments
 * validated on the host before the first HIP call, outputs fully overwritten unless a flag says otherwise, calls only
 * enqueue work on `stream`.  Every call may be captured into a HIP graph.  A call runs on the current device, which must be the one that
 * holds its tensors.  Outputs and workspaces share no memory with an input or with each other, except where an output may be an input
 * itself; calls that break this are refused (SBP_ERR_SHAPE).
 */
#ifndef SBP_LM_H_
#define SBP_LM_H_

#include "sbp.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * Attention whose scores are capped, biased by distance and masked.  Per sample b and query head a, with query i and
 * key j at positions pos_i, pos_j of the sample (kv: the key / value head that query head a reads, a * h_kv / h):
 *   z_ij = scale * q_i.k_j
 *   c_ij = cap * tanh(z_ij / cap)                   (cap = 0: c = z)
 *   s_ij = c_ij - slopes[a] * |pos_i - pos_j|       (slopes = NULL: s = c)
 *   j is visible to i  iff  (not causal, or pos_j <= pos_i, or pos_j < prefix[b])
 *                      and  (doc = NULL, or doc_i = doc_j >= 0)
 *   lse_i = log sum_{visible j} exp(s_ij),          A_i = sum_{visible j} exp(s_ij - lse_i) v_j
 * A row that sees nothing (a token of no document: doc < 0) has A_i = +0 and lse_i = -inf; its gradients are +0.
 * Values of keys that a query does not see never reach its results, not even infinities and NaN.  (Calls on tensors that hold such values
 * take up to some 13 times as long: results that are not finite are computed again without what they do not see.)
 * The backward is "Drop QKV" on the kept tokens (see sbp_backward_attention): i and j run over the kept tokens of the
 * sample only, lse and A come from the forward over all tokens:
 *   P_ij  = exp(s_ij - lse_i) for visible j, else 0
 *   dV_j  = sum_i P_ij dA_i
 *   dM_ij = P_ij (dA_i.v_j - dA_i.A_i) (1 - tanh^2(z_ij / cap))
 *   dQ_i  = scale * sum_j dM_ij k_j,   dK_j = scale * sum_i dM_ij q_i
 * with dK and dV summed over the query heads that share the key / value head.  slopes are constants of the model: no
 * gradient.
 */
typedef struct sbp_attention_desc {
  int32_t  B;             /* samples, >= 1 */
  int32_t  n;             /* tokens per sample, 1 .. 2^24 */
  int32_t  h, h_kv;       /* query heads and key / value heads, h a multiple of h_kv */
  int32_t  d;             /* head dimension: 16, 32, 64 or 128 */
  int32_t  causal;        /* 0 or 1 */
  float    scale;         /* usually 1 / sqrt(d); finite */
  float    cap;           /* 0 .. 1024; 0: scores are not capped */
  const float*   slopes;  /* device, [h] fp32, or NULL */
  const int32_t* doc;     /* device, [B*n] document of every token (any numbers; < 0: of none), or NULL */
  const int32_t* prefix;  /* device, [B] keys at positions below it are visible to all queries of the sample (within the
                             document); only with causal = 1; or NULL */
  /* one call: B * n < 2^31, (h + 2*h_kv) * d <= 2^24, B * h * ceil(n / 32) < 2^22 */
} sbp_attention_desc;

/*
 * Forward over all tokens.
 *   qkv  device, in,  [B*n, (h + 2*h_kv)*d] of `dtype`: q | k | v, each head-major (h = h_kv: the layout of
 *        sbp_backward_attention)
 *   A    device, out, [B*n, h*d] of `dtype`
 *   lse  device, out, [B*n, h] fp32, natural logarithm; or NULL
 * qkv and A 16-byte aligned, A not qkv.  Sums and the softmax statistics are fp32.  In bf16 the weights are rounded to bf16 before the
 * second product: exp(s - a running maximum), or, with 0 < cap <= 60 and no slopes, exp(s) itself, where the row's largest weight is rounded
 * as well (A is divided by the sum of the rounded weights then) and what adds less than 2^-66 to an element of A may be lost; and beyond 32 tokens
 * tanh is good to a few steps of fp32 of 1, so that lse is off by up to 2^-22 cap.  Deterministic.
 */
int32_t sbp_forward_attention_masked(const sbp_attention_desc* desc, const void* qkv, int32_t dtype, void* A, float* lse,
                                     void* stream);

/* Host only.  Bytes of workspace sbp_backward_attention_masked needs (0 on invalid sizes). */
size_t sbp_backward_attention_masked_workspace(const sbp_attention_desc* desc, int32_t n_k, int32_t dtype);

/*
 * Backward on the kept tokens.  Every sample keeps n_k of its n tokens; the tensors hold kept tokens only,
 * sample-major, as sbp_forward_cache gathers them.
 *   idx      device, in, [B*n_k] kept rows: idx[b*n_k + t] = b*n + position, every position of a sample at most once,
 *            in any order (as sbp_sample_indices writes them); NULL: all tokens, n_k = n
 *   qkv_k    device, in, [B*n_k, (h + 2*h_kv)*d]      A_k, dA_k  device, in, [B*n_k, h*d]      lse_k  device, in, [B*n_k, h] fp32
 *   dqkv_k   device, out, [B*n_k, (h + 2*h_kv)*d] of `dtype`: dQ | dK | dV; must not be one of the inputs
 *   workspace  device, 256-byte aligned, sbp_backward_attention_masked_workspace(...) bytes
 * qkv_k, A_k, dA_k, dqkv_k 16-byte aligned.  In bf16 P and dM are rounded to bf16 before the second products.
 * Deterministic.
 */
int32_t sbp_backward_attention_masked(const sbp_attention_desc* desc, const void* qkv_k, const void* A_k, const void* dA_k,
                                      const float* lse_k, const int32_t* idx, int32_t n_k, int32_t dtype, void* dqkv_k,
                                      void* workspace, size_t workspace_bytes, void* stream);

/*
 * The step between two blocks of a network: the norm after a block, its gate, the residual sum, and the norm before the
 * next block, all rows at once:
 *   u     = post(y)                       post(y) = norm(y) * gamma_post + beta_post   (gamma_post = NULL: u = y)
 *   x_out = alpha * x + gate * u          gate [G, C]: row r has gate[r / (M / G)]     (gate = NULL: 1)
 *   z     = pre(x_out)                    pre(x) = norm(x) * gamma_pre + beta_pre
 *   norm over the C channels of a row: SBP_NORM_RMS x / sqrt(mean(x^2) + eps), SBP_NORM_LAYER (x - mean(x)) /
 *   sqrt(var(x) + eps) with the biased variance.
 * z is the norm of the sum before it is rounded to `dtype`.
 */
#define SBP_NORM_RMS   0
#define SBP_NORM_LAYER 1
typedef struct sbp_residual_norm_desc {
  int64_t M;                /* rows of the residual stream */
  int32_t C;                /* channels, 1 .. 16384 */
  int32_t kind;             /* SBP_NORM_RMS or SBP_NORM_LAYER, for both norms */
  int32_t G;                /* rows of gate, M a multiple of it (1: a gate per channel; the batch size: one per sample); >= 1 */
  float   alpha;            /* residual scale; finite */
  float   eps;              /* > 0 */
  uint32_t reserved;        /* 0 */
  const float *gate;        /* device, [G, C] fp32, or NULL */
  const float *gamma_post, *beta_post;   /* device, [C] fp32; gamma NULL: no norm after the block (beta must be NULL as well); beta NULL: 0 */
  const float *gamma_pre, *beta_pre;     /* the same for the next block's norm */
} sbp_residual_norm_desc;

/*
 * Forward.  x, y, x_out, z: device, [M, C] of `dtype`; y NULL: x_out = alpha * x (the norm before the first block;
 * gate and gamma_post must be NULL).  x_out NULL or z NULL (required NULL without gamma_pre) skips that output; x_out
 * may be x or y.
 */
int32_t sbp_forward_residual_norm(const sbp_residual_norm_desc* desc, const void* x, const void* y, int32_t dtype,
                                  void* x_out, void* z, void* stream);

/* Host only.  Bytes of workspace sbp_backward_residual_norm needs (0 on invalid sizes). */
size_t sbp_backward_residual_norm_workspace(const sbp_residual_norm_desc* desc, int64_t K, int32_t dtype, uint32_t flags);

/*
 * Backward on the kept rows.  The residual stream's own gradient passes through every row; the block's branch and the
 * next block's norm have gradients at the kept rows only.  For kept row j, r = idx[j]:
 *   t         = dx_out[r] + pre'(dz_k[j])         gradient of x_out[r] (pre' = 0 if dz_k is NULL, dx_out NULL counts as 0)
 *   dx[r]     = alpha * t;  dropped rows: dx[r] = alpha * dx_out[r]
 *   dy_k[j]   = post'(gate * t)
 *   dgamma_pre = sum_j dz_k xhat_j,  dbeta_pre = sum_j dz_k,  dgate[g] = sum_{j of group g} t * u_j,
 *   dgamma_post = sum_j gate t yhat_j,  dbeta_post = sum_j gate t
 *   dx_out   device, in,  [M, C] of `dtype` ([K, C], row j, with SBP_FLAG_DX_COMPACT), or NULL
 *   dz_k     device, in,  [K, C], or NULL (with it x_out_k and desc->gamma_pre are needed)
 *   x_out_k, y_k  device, in, [K, C] kept rows of x_out and y (y_k may be NULL if dy_k and the gradients of gate, gamma_post and beta_post are not wanted)
 *   idx, inv      as for sbp_backward_linear (idx unused and inv unused with SBP_FLAG_DX_COMPACT; idx may be NULL then).  With
 *            G > 1 every group keeps K / G rows, group-major in idx, as the samplers of this library write them
 *   dx       device, out, [M, C] of `dtype` ([K, C] with SBP_FLAG_DX_COMPACT), or NULL; may be dx_out
 *   dy_k     device, out, [K, C] of `dtype`, or NULL; may be y_k or dz_k
 *   grads    the five parameter gradients, fp32, each may be NULL; added to with SBP_FLAG_ACCUMULATE_DW
 *   flags    SBP_FLAG_DX_COMPACT, SBP_FLAG_ACCUMULATE_DW
 *   workspace  device, 256-byte aligned, sbp_backward_residual_norm_workspace(...) bytes
 * fp32 arithmetic, sums over rows in a fixed order.
 */
typedef struct sbp_residual_norm_grads {
  float *dgate;                        /* [G, C] */
  float *dgamma_post, *dbeta_post, *dgamma_pre, *dbeta_pre;   /* [C] */
} sbp_residual_norm_grads;
int32_t sbp_backward_residual_norm(const sbp_residual_norm_desc* desc, const void* dx_out, const void* dz_k, const void* x_out_k,
                                   const void* y_k, const int32_t* idx, const int32_t* inv, int64_t K, int32_t dtype,
                                   void* dx, void* dy_k, const sbp_residual_norm_grads* grads, void* workspace,
                                   size_t workspace_bytes, uint32_t flags, void* stream);

/*
 * Token table.  Forward: E[r, :] = scale * table[tokens[r], :], rounded once; a token outside [0, V) gives a row of +0.
 *   tokens  device, in, [M] int32 (token_bytes = 4) or int64 (token_bytes = 8)
 *   table   device, in, [V, C] of `dtype`;   E  device, out, [M, C] of `dtype`
 * M < 2^31, V < 2^30, C <= 2^30.
 */
int32_t sbp_forward_embedding(const void* tokens, int32_t token_bytes, const void* table, int64_t M, int64_t V, int32_t C,
                              float scale, int32_t dtype, void* E, void* stream);

/* Host only.  Bytes of workspace sbp_backward_embedding needs (0 on invalid sizes). */
size_t sbp_backward_embedding_workspace(int64_t M, int64_t K, int64_t V, int32_t C, int32_t dtype, uint32_t flags);

/*
 * Gradient of the table from the kept rows: dtable[v, :] = scale * sum over the kept rows j with tokens[idx[j]] = v of
 * dE[idx[j], :], every other row +0.  The kept rows are sorted by token (stable), so that sums run in the order of idx:
 * deterministic, no atomics on floating-point values.
 *   dE      device, in, [M, C] of `dtype` (only rows in idx are read), or [K, C] with SBP_FLAG_DY_COMPACT
 *   tokens  device, in, [M]
 *   idx     device, in, [K] row ids in [0, M), or NULL: all rows, K = M
 *   dtable  device, out, [V, C] fp32 (bf16 with SBP_FLAG_DW_OUT_BF16: the fp32 sum rounded once); SBP_FLAG_ACCUMULATE_DW
 *           adds to the rows of the tokens that occur and leaves the others as they are (the gradient of a table that is
 *           also the output projection's weight)
 *   flags   SBP_FLAG_DY_COMPACT, SBP_FLAG_ACCUMULATE_DW, SBP_FLAG_DW_OUT_BF16
 *   workspace  device, 256-byte aligned, sbp_backward_embedding_workspace(...) bytes
 * K < 2^30, V < 2^30, C <= 2^30, K * C < 2^37.
 */
int32_t sbp_backward_embedding(const void* dE, const void* tokens, int32_t token_bytes, const int32_t* idx, int64_t M, int64_t K,
                               int64_t V, int32_t C, float scale, int32_t dtype, void* dtable, void* workspace,
                               size_t workspace_bytes, uint32_t flags, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* SBP_LM_H_ */
