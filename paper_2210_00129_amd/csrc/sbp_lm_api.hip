// C ABI of the language-model steps (sbp_lm.h): host-side validation, then kernel launches.  Every argument check runs before
// the first HIP call, so that error paths need no device.
#include <algorithm>
#include <cmath>
#include <initializer_list>

#include "sbp_lm_internal.h"

namespace sbp {

static bool known_dtype(int32_t dtype) { return dtype == SBP_F32 || dtype == SBP_BF16; }

static int32_t check_workspace(const void* ws, size_t have, size_t need) {
  if (need == 0) return SBP_OK;
  if (!ws || have < need || reinterpret_cast<uintptr_t>(ws) % 256)
    return fail(SBP_ERR_WORKSPACE, "workspace missing, misaligned or smaller than %zu bytes", need);
  return SBP_OK;
}

// A tensor of a call; an output may be one of two inputs itself (`same`), element for element.
struct Range {
  const char* name;
  const void* p;
  size_t bytes;
  const void* same[2] = {nullptr, nullptr};
};
static bool overlap(const Range& a, const Range& b) {
  const uintptr_t x = (uintptr_t)a.p, y = (uintptr_t)b.p;
  return x && y && a.bytes && b.bytes && x < y + b.bytes && y < x + a.bytes;
}
// Outputs (the workspace is one) share no memory with an input nor with each other: the workgroups of a launch run in any order.
static int32_t check_overlap(std::initializer_list<Range> outs, std::initializer_list<Range> ins) {
  for (const Range* o = outs.begin(); o != outs.end(); ++o) {
    for (const Range& i : ins)
      if (overlap(*o, i) && !(o->p == i.p && (o->p == o->same[0] || o->p == o->same[1]))) return fail(SBP_ERR_SHAPE, "%s and %s overlap", o->name, i.name);
    for (const Range* q = outs.begin(); q != o; ++q)
      if (overlap(*o, *q)) return fail(SBP_ERR_SHAPE, "%s and %s overlap", o->name, q->name);
  }
  return SBP_OK;
}
static size_t elem_bytes(int32_t dtype) { return dtype == SBP_F32 ? 4 : 2; }

// rows: tokens per sample in the tensors
static int32_t validate_masked(const sbp_attention_desc* a, int64_t rows, int32_t dtype) {
  if (!a) return fail(SBP_ERR_NULL, "attention descriptor is NULL");
  if (!known_dtype(dtype)) return fail(SBP_ERR_DTYPE, "unknown dtype %d", dtype);
  if (a->B < 1 || a->n < 1 || a->h < 1 || a->h_kv < 1 || a->h % a->h_kv)
    return fail(SBP_ERR_SHAPE, "bad shape B=%d n=%d h=%d h_kv=%d (h must be a multiple of h_kv)", a->B, a->n, a->h, a->h_kv);
  if (a->d != 16 && a->d != 32 && a->d != 64 && a->d != 128) return fail(SBP_ERR_SHAPE, "head dimension must be 16, 32, 64 or 128, got %d", a->d);
  if ((int64_t)a->B * a->n > INT32_MAX) return fail(SBP_ERR_SHAPE, "B*n=%lld exceeds int32 row ids", (long long)a->B * a->n);
  if ((a->h + 2LL * a->h_kv) * a->d > (1 << 24)) return fail(SBP_ERR_SHAPE, "(h + 2 h_kv) * d is too large");
  if (a->n > (1 << 24)) return fail(SBP_ERR_SHAPE, "n=%d: positions beyond 2^24 are not exact in fp32", a->n);
  if (rows < 0 || rows > a->n) return fail(SBP_ERR_SHAPE, "need 0 <= n_k <= n, got n_k=%lld n=%d", (long long)rows, a->n);
  // (a grid of 256 or 512 threads per 32 tokens and head, in two roles, stays below 2^32 threads; and the four tables of the backward's
  // workspace, 4 bytes per token and head of samples padded to 64 tokens, below 2^32 bytes together: its kernel's offsets into them are 32 bits)
  if ((int64_t)a->B * a->h * ceil_div(a->n, 32) >= (1 << 22)) return fail(SBP_ERR_SHAPE, "B * h * n is too large for one call");
  if (a->causal != 0 && a->causal != 1) return fail(SBP_ERR_FLAGS, "causal must be 0 or 1, got %d", a->causal);
  if (!std::isfinite(a->scale)) return fail(SBP_ERR_SHAPE, "scale must be finite");
  // (the bf16 kernels take tanh from one exponential and a reciprocal, to a few steps of fp32 of 1: the capped score is then off by up to
  // 2^-22 cap, which for 1024 is still 2^-4 of the rounding of a weight to bf16)
  if (!(a->cap >= 0.f && a->cap <= 1024.f)) return fail(SBP_ERR_SHAPE, "cap must be 0 or up to 1024");
  if (a->prefix && !a->causal) return fail(SBP_ERR_FLAGS, "prefix needs causal = 1");
  return SBP_OK;
}

static MaskedAttention masked_args(const sbp_attention_desc& d, int rows) {
  MaskedAttention a = {};
  a.slopes = d.slopes; a.doc = d.doc; a.prefix = d.prefix;
  a.B = d.B; a.n = d.n; a.rows = rows; a.h = d.h; a.hk = d.h_kv; a.d = d.d; a.causal = d.causal;
  a.scale = d.scale; a.cap = d.cap;
  a.per_cap = d.cap > 0.f ? std::min(std::max(d.scale / d.cap, -1e38f), 1e38f) : 0.f;
  return a;
}

static int32_t validate_residual(const sbp_residual_norm_desc* a, int32_t dtype) {
  if (!a) return fail(SBP_ERR_NULL, "norm descriptor is NULL");
  if (!known_dtype(dtype)) return fail(SBP_ERR_DTYPE, "unknown dtype %d", dtype);
  if (a->M < 1 || a->M > INT32_MAX || a->C < 1 || a->C > 16384)
    return fail(SBP_ERR_SHAPE, "bad shape M=%lld C=%d (1 <= C <= 16384)", (long long)a->M, a->C);
  if (a->kind != SBP_NORM_RMS && a->kind != SBP_NORM_LAYER) return fail(SBP_ERR_FLAGS, "unknown kind of norm %d", a->kind);
  if (a->reserved) return fail(SBP_ERR_FLAGS, "reserved must be 0");
  if (a->G < 1 || a->M % a->G) return fail(SBP_ERR_SHAPE, "M=%lld must be a multiple of G=%d >= 1", (long long)a->M, a->G);
  if (a->G > 65535) return fail(SBP_ERR_SHAPE, "G=%d is larger than 65535", a->G);
  if (!std::isfinite(a->alpha)) return fail(SBP_ERR_SHAPE, "alpha must be finite");
  if (!(a->eps > 0.f) || !std::isfinite(a->eps)) return fail(SBP_ERR_SHAPE, "eps must be positive and finite");
  if ((a->beta_post && !a->gamma_post) || (a->beta_pre && !a->gamma_pre)) return fail(SBP_ERR_NULL, "beta without gamma");
  return SBP_OK;
}

static int32_t validate_residual_backward(const sbp_residual_norm_desc* a, int64_t K, int32_t dtype, uint32_t flags) {
  const int32_t st = validate_residual(a, dtype);
  if (st != SBP_OK) return st;
  if (flags & ~(SBP_FLAG_DX_COMPACT | SBP_FLAG_ACCUMULATE_DW)) return fail(SBP_ERR_FLAGS, "unknown flags 0x%x", flags);
  if (K < 0 || K > a->M) return fail(SBP_ERR_SHAPE, "need 0 <= K <= M, got K=%lld M=%lld", (long long)K, (long long)a->M);
  if (K % a->G) return fail(SBP_ERR_SHAPE, "K=%lld must be a multiple of G=%d", (long long)K, a->G);
  return SBP_OK;
}

static int32_t validate_embedding(int64_t M, int64_t V, int32_t C, float scale, int32_t token_bytes, int32_t dtype) {
  if (!known_dtype(dtype)) return fail(SBP_ERR_DTYPE, "unknown dtype %d", dtype);
  if (token_bytes != 4 && token_bytes != 8) return fail(SBP_ERR_DTYPE, "token_bytes must be 4 or 8, got %d", token_bytes);
  if (M < 0 || M > INT32_MAX || V < 1 || V >= (1 << 30) || C < 1) return fail(SBP_ERR_SHAPE, "bad shape M=%lld V=%lld C=%d", (long long)M, (long long)V, C);
  // (a lane's next column, up to 2048 on, and a slice's end stay below 2^31)
  if (C > (1 << 30)) return fail(SBP_ERR_SHAPE, "C=%d is larger than 2^30", C);
  if (!std::isfinite(scale)) return fail(SBP_ERR_SHAPE, "scale must be finite");
  return SBP_OK;
}

static int32_t validate_embedding_backward(int64_t M, int64_t K, int64_t V, int32_t C, int32_t token_bytes, int32_t dtype, uint32_t flags) {
  const int32_t st = validate_embedding(M, V, C, 1.f, token_bytes, dtype);
  if (st != SBP_OK) return st;
  if (flags & ~(SBP_FLAG_DY_COMPACT | SBP_FLAG_ACCUMULATE_DW | SBP_FLAG_DW_OUT_BF16)) return fail(SBP_ERR_FLAGS, "unknown flags 0x%x", flags);
  if (K < 0 || K > M || K >= (1 << 30)) return fail(SBP_ERR_SHAPE, "need 0 <= K <= M, K < 2^30, got K=%lld M=%lld", (long long)K, (long long)M);
  // (a wavefront per 32 rows and 64 columns stays below 2^32 threads)
  if (ceil_div(K, 32) * ceil_div(C, 64) >= (1 << 26)) return fail(SBP_ERR_SHAPE, "K * C is too large for one call");
  return SBP_OK;
}

}  // namespace sbp

using namespace sbp;

extern "C" {

int32_t sbp_forward_attention_masked(const sbp_attention_desc* desc, const void* qkv, int32_t dtype, void* A, float* lse, void* stream) {
  int32_t st = validate_masked(desc, 0, dtype);
  if (st != SBP_OK) return st;
  if (!qkv || !A) return fail(SBP_ERR_NULL, "qkv or A is NULL");
  if (((uintptr_t)qkv | (uintptr_t)A) & 15) return fail(SBP_ERR_SHAPE, "tensors must be 16-byte aligned");
  if (A == qkv) return fail(SBP_ERR_SHAPE, "A must not be qkv");
  const size_t rows = (size_t)desc->B * desc->n, size = elem_bytes(dtype);
  st = check_overlap({{"A", A, rows * desc->h * desc->d * size}, {"lse", lse, rows * desc->h * 4}},
                     {{"qkv", qkv, rows * (desc->h + 2 * (size_t)desc->h_kv) * desc->d * size}, {"slopes", desc->slopes, (size_t)desc->h * 4},
                      {"doc", desc->doc, rows * 4}, {"prefix", desc->prefix, (size_t)desc->B * 4}});
  if (st != SBP_OK) return st;
  MaskedAttention a = masked_args(*desc, desc->n);
  a.qkv = qkv; a.out = A; a.lse_out = lse;
  return launch_forward_attention_masked(a, dtype, static_cast<hipStream_t>(stream));
}

size_t sbp_backward_attention_masked_workspace(const sbp_attention_desc* desc, int32_t n_k, int32_t dtype) {
  if (validate_masked(desc, n_k, dtype) != SBP_OK) return 0;
  return plan_masked_attention_backward(*desc, n_k, dtype).bytes;
}

int32_t sbp_backward_attention_masked(const sbp_attention_desc* desc, const void* qkv_k, const void* A_k, const void* dA_k, const float* lse_k,
                                      const int32_t* idx, int32_t n_k, int32_t dtype, void* dqkv_k, void* ws, size_t ws_bytes, void* stream) {
  int32_t st = validate_masked(desc, n_k, dtype);
  if (st != SBP_OK) return st;
  if (n_k == 0) return SBP_OK;   // no kept token (empty tensors may have NULL storage)
  if (!idx && n_k != desc->n) return fail(SBP_ERR_NULL, "idx is NULL but n_k=%d is not n=%d", n_k, desc->n);
  if (!qkv_k || !A_k || !dA_k || !lse_k || !dqkv_k) return fail(SBP_ERR_NULL, "qkv_k, A_k, dA_k, lse_k or dqkv_k is NULL");
  if (((uintptr_t)qkv_k | (uintptr_t)A_k | (uintptr_t)dA_k | (uintptr_t)dqkv_k) & 15) return fail(SBP_ERR_SHAPE, "tensors must be 16-byte aligned");
  if (dqkv_k == qkv_k || dqkv_k == A_k || dqkv_k == dA_k) return fail(SBP_ERR_SHAPE, "dqkv_k must not be one of the inputs");
  const MaskedAttentionPlan p = plan_masked_attention_backward(*desc, n_k, dtype);
  st = check_workspace(ws, ws_bytes, p.bytes);
  if (st != SBP_OK) return st;
  const size_t rows = (size_t)desc->B * n_k, size = elem_bytes(dtype), out = rows * desc->h * desc->d * size,
               all = rows * (desc->h + 2 * (size_t)desc->h_kv) * desc->d * size;
  st = check_overlap({{"dqkv_k", dqkv_k, all}, {"the workspace", ws, p.bytes}},
                     {{"qkv_k", qkv_k, all}, {"A_k", A_k, out}, {"dA_k", dA_k, out}, {"lse_k", lse_k, rows * desc->h * 4}, {"idx", idx, rows * 4},
                      {"slopes", desc->slopes, (size_t)desc->h * 4}, {"doc", desc->doc, (size_t)desc->B * desc->n * 4},
                      {"prefix", desc->prefix, (size_t)desc->B * 4}});
  if (st != SBP_OK) return st;
  MaskedAttention a = masked_args(*desc, n_k);
  a.qkv = qkv_k; a.A = A_k; a.dA = dA_k; a.lse = lse_k; a.idx = idx; a.out = dqkv_k;
  return launch_backward_attention_masked(a, p, dtype, ws, static_cast<hipStream_t>(stream));
}

int32_t sbp_forward_residual_norm(const sbp_residual_norm_desc* desc, const void* x, const void* y, int32_t dtype, void* x_out, void* z,
                                  void* stream) {
  int32_t st = validate_residual(desc, dtype);
  if (st != SBP_OK) return st;
  if (!x) return fail(SBP_ERR_NULL, "x is NULL");
  if (!y && (desc->gate || desc->gamma_post)) return fail(SBP_ERR_NULL, "y is NULL but gate or gamma_post is given");
  if (z && !desc->gamma_pre) return fail(SBP_ERR_NULL, "gamma_pre is NULL but z is requested");
  if (z && (z == x || z == y || z == x_out)) return fail(SBP_ERR_SHAPE, "z must be a buffer of its own");
  if (!x_out && !z) return SBP_OK;
  const size_t all = (size_t)desc->M * desc->C * elem_bytes(dtype), c = (size_t)desc->C * 4;
  st = check_overlap({{"x_out", x_out, all, {x, y}}, {"z", z, all}},
                     {{"x", x, all}, {"y", y, all}, {"gate", desc->gate, desc->G * c}, {"gamma_post", desc->gamma_post, c}, {"beta_post", desc->beta_post, c},
                      {"gamma_pre", desc->gamma_pre, c}, {"beta_pre", desc->beta_pre, c}});
  if (st != SBP_OK) return st;
  return launch_forward_residual_norm(*desc, x, y, dtype, x_out, z, static_cast<hipStream_t>(stream));
}

size_t sbp_backward_residual_norm_workspace(const sbp_residual_norm_desc* desc, int64_t K, int32_t dtype, uint32_t flags) {
  if (validate_residual_backward(desc, K, dtype, flags) != SBP_OK) return 0;
  return plan_residual_norm_backward(*desc, K, dtype, flags).bytes;
}

int32_t sbp_backward_residual_norm(const sbp_residual_norm_desc* desc, const void* dx_out, const void* dz_k, const void* x_out_k, const void* y_k,
                                   const int32_t* idx, const int32_t* inv, int64_t K, int32_t dtype, void* dx, void* dy_k,
                                   const sbp_residual_norm_grads* grads, void* ws, size_t ws_bytes, uint32_t flags, void* stream) {
  int32_t st = validate_residual_backward(desc, K, dtype, flags);
  if (st != SBP_OK) return st;
  const sbp_residual_norm_grads g = grads ? *grads : sbp_residual_norm_grads{};
  const bool compact = flags & SBP_FLAG_DX_COMPACT;
  if (dz_k && K > 0 && (!x_out_k || !desc->gamma_pre)) return fail(SBP_ERR_NULL, "dz_k needs x_out_k and gamma_pre");
  if ((g.dgamma_pre || g.dbeta_pre) && (!desc->gamma_pre || (!dz_k && K > 0))) return fail(SBP_ERR_NULL, "dgamma_pre and dbeta_pre need gamma_pre and dz_k");
  if ((g.dgamma_post || g.dbeta_post) && !desc->gamma_post) return fail(SBP_ERR_NULL, "dgamma_post and dbeta_post need gamma_post");
  if (g.dgate && !desc->gate) return fail(SBP_ERR_NULL, "dgate needs gate");
  if (K > 0 && !y_k && (g.dgate || g.dgamma_post || g.dbeta_post || (dy_k && desc->gamma_post))) return fail(SBP_ERR_NULL, "y_k is NULL");
  const bool rows = !compact && (dx || dx_out);
  if (rows && !idx && K > 0) return fail(SBP_ERR_NULL, "idx is NULL");
  if (dy_k && (dy_k == dx_out || dy_k == dx || dy_k == x_out_k)) return fail(SBP_ERR_SHAPE, "dy_k must not be dx_out, dx or x_out_k");
  if (dx && (dx == dz_k || dx == x_out_k || dx == y_k)) return fail(SBP_ERR_SHAPE, "dx must not be dz_k, x_out_k or y_k");
  const ResidualNormPlan p = plan_residual_norm_backward(*desc, K, dtype, flags);
  st = check_workspace(ws, ws_bytes, p.bytes);
  if (st != SBP_OK) return st;
  const size_t c = (size_t)desc->C * 4, kept = (size_t)K * desc->C * elem_bytes(dtype), all = compact ? kept : (size_t)desc->M * desc->C * elem_bytes(dtype);
  st = check_overlap({{"dx", dx, all, {dx_out, nullptr}}, {"dy_k", dy_k, kept, {y_k, dz_k}}, {"dgate", g.dgate, desc->G * c}, {"dgamma_post", g.dgamma_post, c},
                      {"dbeta_post", g.dbeta_post, c}, {"dgamma_pre", g.dgamma_pre, c}, {"dbeta_pre", g.dbeta_pre, c}, {"the workspace", ws, p.bytes}},
                     {{"dx_out", dx_out, all}, {"dz_k", dz_k, kept}, {"x_out_k", x_out_k, kept}, {"y_k", y_k, kept}, {"idx", compact ? nullptr : idx, (size_t)K * 4},
                      {"inv", compact ? nullptr : inv, (size_t)desc->M * 4}, {"gate", desc->gate, desc->G * c}, {"gamma_post", desc->gamma_post, c},
                      {"beta_post", desc->beta_post, c}, {"gamma_pre", desc->gamma_pre, c}, {"beta_pre", desc->beta_pre, c}});
  if (st != SBP_OK) return st;
  return launch_backward_residual_norm(p, *desc, dx_out, dz_k, x_out_k, y_k, idx, inv, K, dtype, dx, dy_k, g, ws, flags,
                                       static_cast<hipStream_t>(stream));
}

int32_t sbp_forward_embedding(const void* tokens, int32_t token_bytes, const void* table, int64_t M, int64_t V, int32_t C, float scale,
                              int32_t dtype, void* E, void* stream) {
  int32_t st = validate_embedding(M, V, C, scale, token_bytes, dtype);
  if (st != SBP_OK) return st;
  if (M == 0) return SBP_OK;
  if (!tokens || !table || !E) return fail(SBP_ERR_NULL, "tokens, table or E is NULL");
  if ((uintptr_t)tokens % token_bytes) return fail(SBP_ERR_SHAPE, "tokens must be aligned to their size");
  const size_t row = (size_t)C * elem_bytes(dtype);
  st = check_overlap({{"E", E, M * row}}, {{"tokens", tokens, (size_t)M * token_bytes}, {"table", table, V * row}});
  if (st != SBP_OK) return st;
  return launch_forward_embedding(tokens, token_bytes, table, M, V, C, scale, dtype, E, static_cast<hipStream_t>(stream));
}

size_t sbp_backward_embedding_workspace(int64_t M, int64_t K, int64_t V, int32_t C, int32_t dtype, uint32_t flags) {
  if (validate_embedding_backward(M, K, V, C, 4, dtype, flags) != SBP_OK) return 0;
  return plan_embedding_backward(K, V, C, flags).bytes;
}

int32_t sbp_backward_embedding(const void* dE, const void* tokens, int32_t token_bytes, const int32_t* idx, int64_t M, int64_t K, int64_t V,
                               int32_t C, float scale, int32_t dtype, void* dtable, void* ws, size_t ws_bytes, uint32_t flags, void* stream) {
  int32_t st = validate_embedding_backward(M, K, V, C, token_bytes, dtype, flags);
  if (st != SBP_OK) return st;
  if (!std::isfinite(scale)) return fail(SBP_ERR_SHAPE, "scale must be finite");
  if (!dtable) return fail(SBP_ERR_NULL, "dtable is NULL");
  if (K > 0 && (!dE || !tokens)) return fail(SBP_ERR_NULL, "dE or tokens is NULL");
  if (!idx && K > 0 && K != M) return fail(SBP_ERR_NULL, "idx is NULL but K=%lld is not M=%lld", (long long)K, (long long)M);
  if ((uintptr_t)tokens % token_bytes) return fail(SBP_ERR_SHAPE, "tokens must be aligned to their size");
  const EmbeddingPlan p = plan_embedding_backward(K, V, C, flags);
  st = check_workspace(ws, ws_bytes, p.bytes);
  if (st != SBP_OK) return st;
  st = check_overlap({{"dtable", dtable, (size_t)V * C * (flags & SBP_FLAG_DW_OUT_BF16 ? 2 : 4)}, {"the workspace", ws, p.bytes}},
                     {{"dE", dE, (size_t)(flags & SBP_FLAG_DY_COMPACT ? K : M) * C * elem_bytes(dtype)}, {"tokens", tokens, (size_t)M * token_bytes},
                      {"idx", idx, (size_t)K * 4}});
  if (st != SBP_OK) return st;
  return launch_backward_embedding(p, dE, tokens, token_bytes, idx, M, K, V, C, scale, dtype, dtable, ws, flags,
                                   static_cast<hipStream_t>(stream));
}

}  // extern "C"
