"""The steps of a language model's block between its linear layers, and the token table below the first block
(include/sbp_lm.h).  Re-exported by the package:

    A, lse  = forward_attention_masked(qkv, B, h, d, scale, causal=True, cap=50.0, doc=doc)     # all tokens
    dqkv_k  = backward_attention_masked(qkv_k, A_k, dA_k, lse_k, B, h, d, scale, n=n, idx=idx, causal=True, ...)
    x, z    = forward_residual_norm(x, y, gamma_post=g1, gamma_pre=g2)      # post-norm, gate, residual sum, pre-norm
    grads   = backward_residual_norm(dx, dz_k, x_k, y_k, idx, M, gamma_post=g1, gamma_pre=g2)
    E       = forward_embedding(tokens, table, scale)
    dtable  = backward_embedding(dE, tokens, V, idx=idx, scale=scale)

Like the rest of the binding: arguments are checked, outputs and workspaces allocated, the work runs in the library's
kernels on the current stream of the tensors' device (all of a call's tensors live on one).
"""
from __future__ import annotations

from . import _lib

NORM_RMS, NORM_LAYER = 0, 1


def _native():
    return _lib._native_lm or _lib.native_lm()


def forward_attention_masked(qkv, B, h, d, scale, h_kv=None, cap=0.0, causal=False, slopes=None, doc=None, prefix=None, out=None,
                             lse_out=None):
    """Attention over all tokens of every sample.  qkv [B*n, (h + 2*h_kv)*d] = q | k | v (h_kv None: h).
    cap > 0: scores cap * tanh(score / cap); slopes fp32 [h]: minus slope * distance; causal; prefix int32 [B]: keys before it are
    seen by every query of the sample; doc int32 [B*n]: a token sees its own document only, a negative number is padding.
    Returns (A [B*n, h*d], lse fp32 [B*n, h]); rows that see nothing are +0 with lse -inf."""
    return _native().attention_forward(qkv, B, h, d, scale, h_kv, cap, causal, slopes, doc, prefix, out, lse_out)


def backward_attention_masked(qkv_k, A_k, dA_k, lse_k, B, h, d, scale, n=None, idx=None, h_kv=None, cap=0.0, causal=False, slopes=None,
                              doc=None, prefix=None, out=None, workspace=None):
    """Its backward on the kept tokens ("Drop QKV").  qkv_k [B*n_k, (h + 2*h_kv)*d], A_k, dA_k [B*n_k, h*d], lse_k fp32 [B*n_k, h]
    are the kept rows idx (int32 [B*n_k], sample-major; None: all tokens) of the forward's n tokens per sample; doc and prefix as
    in the forward.  Returns dqkv_k [B*n_k, (h + 2*h_kv)*d] (dQ | dK | dV)."""
    return _native().attention_backward(qkv_k, A_k, dA_k, lse_k, B, h, d, scale, h_kv, cap, causal, slopes, doc, prefix, n, idx, out, workspace)


def forward_residual_norm(x, y=None, gate=None, alpha=1.0, gamma_post=None, beta_post=None, gamma_pre=None, beta_pre=None, kind=NORM_RMS,
                          eps=1e-5, x_out=None, z=None):
    """x_out = alpha * x + gate * post(y), z = pre(x_out): the norm after a block, its gate, the residual sum and the next block's norm.
    x, y [M, C]; gate fp32 [C] or [G, C] (row r has gate[r // (M / G)]); gammas, betas fp32 [C], gamma None: that norm is left out.
    Returns (x_out, z); z is None without gamma_pre.  x_out may be x (in place)."""
    return _native().norm_forward(x, y, gate, alpha, gamma_post, beta_post, gamma_pre, beta_pre, kind, eps, x_out, z)


def backward_residual_norm(dx_out, dz_k, x_out_k, y_k, idx, M, gate=None, alpha=1.0, gamma_post=None, beta_post=None, gamma_pre=None,
                           kind=NORM_RMS, eps=1e-5, inv=None, flags=0, want=None, dx=None, dy_k=None, grads=None, workspace=None):
    """Backward of forward_residual_norm on the kept rows idx.  dx_out [M, C] (the residual stream's gradient; None: 0), dz_k, x_out_k,
    y_k [K, C].  Returns a dict with the entries named in `want`: dx [M, C] (alpha * dx_out in the dropped rows), dy_k [K, C], and fp32
    dgate, dgamma_post, dbeta_post, dgamma_pre, dbeta_pre; by default dx, dy_k and the gradients of the vectors given (dgamma_pre where
    dz_k is).  FLAG_DX_COMPACT: dx_out and dx are [K, C].  `grads`: preallocated parameter gradients by name (needed with
    FLAG_ACCUMULATE_DW)."""
    return _native().norm_backward(dx_out, dz_k, x_out_k, y_k, idx, M, gate, alpha, gamma_post, beta_post, gamma_pre, None, kind, eps, inv, flags,
                                   want, dx, dy_k, grads, workspace)


def forward_embedding(tokens, table, scale=1.0, out=None):
    """E[r] = scale * table[tokens[r]]: [*tokens.shape, C]; tokens int32 or int64, one outside the table gives a row of +0."""
    return _native().embedding_forward(tokens, table, scale, out)


def backward_embedding(dE, tokens, V, idx=None, scale=1.0, flags=0, dtable=None, workspace=None):
    """dtable [V, C] fp32 (bf16 with FLAG_DW_OUT_BF16) from the kept rows idx (int32 [K]; None: all): scale * the sum of the rows of dE
    whose token it is, +0 elsewhere.  dE [M, C], or [K, C] with FLAG_DY_COMPACT; tokens [M] int32 or int64.  FLAG_ACCUMULATE_DW adds to
    the given dtable and touches no other row."""
    return _native().embedding_backward(dE, tokens, V, idx, scale, flags, dtable, workspace)
