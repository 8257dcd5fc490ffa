// Internal declarations of the language-model steps (sbp_lm.h), beside sbp_internal.h.
#ifndef SBP_LM_INTERNAL_H_
#define SBP_LM_INTERNAL_H_

#include "sbp_internal.h"
#include "sbp_lm.h"

namespace sbp {

// ---- masked attention --------------------------------------------------------------------------
// What every kernel of it is handed: the tensors hold `rows` tokens per sample (all n of them, or the n_k kept ones).
struct MaskedAttention {
  const void *qkv, *A, *dA;
  const float* lse;
  const int32_t* idx;            // kept rows, or NULL: token t of a sample is at position t
  const float* slopes;
  const int32_t* doc;
  const int32_t* prefix;
  void* out;                     // A or dqkv
  float* lse_out;
  int B, n, rows, h, hk, d, causal;
  float scale, cap;
  float per_cap;                 // scale / cap, the factor of q.k under the tanh: finite for the smallest caps too, where 0 times an infinity would be no score
};
struct MaskedAttentionPlan {     // workspace of the backward
  int    npad, nchunks;          // kept tokens per sample in whole tiles; chunks of own tokens per workgroup
  int    parts;                  // workgroups that share a key / value head's query heads
  size_t off_l2, off_nd, off_pos, off_doc, off_range, off_part, bytes;
};
struct LmTables;
MaskedAttentionPlan plan_masked_attention_backward(const sbp_attention_desc& a, int32_t n_k, int32_t dtype);
template <int D> void launch_masked_forward_bf16(const MaskedAttention& a, hipStream_t s);
template <int D> void launch_masked_backward_bf16(const MaskedAttention& a, const LmTables& w, hipStream_t s);
void launch_masked_f32(const MaskedAttention& a, const LmTables* w, hipStream_t s);        // w: backward
int32_t launch_forward_attention_masked(const MaskedAttention& a, int32_t dtype, hipStream_t s);
int32_t launch_backward_attention_masked(const MaskedAttention& a, const MaskedAttentionPlan& p, int32_t dtype, void* ws, hipStream_t s);

// ---- norms between blocks ----------------------------------------------------------------------
struct ResidualNormPlan {
  int    nblocks;                // workgroups per group of rows, and partial sums of each parameter gradient
  size_t off_partial;            // fp32 [G][nblocks][2 or 4][C]
  size_t off_inv;                // int32 [M]
  size_t bytes;
};
ResidualNormPlan plan_residual_norm_backward(const sbp_residual_norm_desc& a, int64_t K, int32_t dtype, uint32_t flags);
int32_t launch_forward_residual_norm(const sbp_residual_norm_desc& a, const void* x, const void* y, int32_t dtype, void* x_out, void* z,
                                     hipStream_t s);
int32_t launch_backward_residual_norm(const ResidualNormPlan& p, const sbp_residual_norm_desc& a, const void* dx_out, const void* dz,
                                      const void* x_out, const void* y, const int32_t* idx, const int32_t* inv, int64_t K, int32_t dtype,
                                      void* dx, void* dy, const sbp_residual_norm_grads& g, void* ws, uint32_t flags, hipStream_t s);

// ---- token table -------------------------------------------------------------------------------
struct EmbeddingPlan {
  bool    sorted;                // else every wavefront looks through the kept tokens for its own table rows
  bool    one;                   // sort: one workgroup, in registers and LDS
  int     nblocks;               // sort: workgroups, each over a run of `per` kept rows
  int64_t per;
  int     passes, bits;          // sort: digits and bits of one
  int     chunks;                // runs of sorted rows that one wavefront sums
  size_t  off_keys[2], off_rows[2], off_hist, off_partial, bytes;
};
EmbeddingPlan plan_embedding_backward(int64_t K, int64_t V, int32_t C, uint32_t flags);
int32_t launch_forward_embedding(const void* tokens, int32_t token_bytes, const void* table, int64_t M, int64_t V, int32_t C, float scale,
                                 int32_t dtype, void* E, hipStream_t s);
int32_t launch_backward_embedding(const EmbeddingPlan& p, const void* dE, const void* tokens, int32_t token_bytes, const int32_t* idx,
                                  int64_t M, int64_t K, int64_t V, int32_t C, float scale, int32_t dtype, void* dtable, void* ws,
                                  uint32_t flags, hipStream_t s);

}  // namespace sbp
#endif
