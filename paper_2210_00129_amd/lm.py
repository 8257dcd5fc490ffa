"""The steps of a language model's block between its linear layers, and the token table below the first block
(include/sbp_lm.h).  Re-exported by the package:

    A, lse  = forward_attention_masked(qkv, B, h, d, scale, causal=True, cap=50.0, doc=doc)     # all tokens
    dqkv_k  = backward_attention_masked(qkv_k, A_k, dA_k, lse_k, B, h, d, scale, n=n, idx=idx, causal=True, ...)
    x, z    = forward_residual_norm(x, y, gamma_post=g1, gamma_pre=g2)      # post-norm, gate, residual sum, pre-norm
    grads   = backward_residual_norm(dx, dz_k, x_k, y_k, idx, M, gamma_post=g1, gamma_pre=g2)
    E       = forward_embedding(tokens, table, scale)
    dtable  = backward_embedding(dE, tokens, V, idx=idx, scale=scale)

Like the rest of the binding: arguments are checked, outputs and workspaces allocated, the work runs in the library's
kernels on the current stream of the tensors' device.
"""
from __future__ import annotations

import ctypes

import torch

from . import _lib
from ._lib import AttentionDesc, ResidualNormDesc, ResidualNormGrads

NORM_RMS, NORM_LAYER = 0, 1
_FLAG_DY_COMPACT, _FLAG_DX_COMPACT, _FLAG_ACCUMULATE, _FLAG_OUT_BF16 = 1, 2, 4, 8
_CODES = {torch.float32: 0, torch.bfloat16: 1}


def _code(t) -> int:
    try:
        return _CODES[t.dtype]
    except KeyError:
        raise TypeError(f"unsupported dtype {t.dtype}; use float32 or bfloat16") from None


def _ptr(t, name, shape, dtype, device):
    """Address of a tensor (None: NULL) that has to be contiguous, on `device`, of this shape and type."""
    if t is None:
        return None
    if not t.is_cuda:
        raise ValueError(f"{name} must live in GPU memory")
    if t.device != device:
        raise ValueError(f"{name} is on {t.device}, not on {device}")
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} must have shape {tuple(shape)}, got {tuple(t.shape)}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return t.data_ptr()


def _call(name, device, *args):
    """One call of the library on the current stream of `device`, which becomes the current device for its duration."""
    fn = getattr(_lib.lib(), name)
    if torch._C._cuda_getDevice() == device.index:
        return _lib.check(fn(*args, torch._C._cuda_getCurrentRawStream(device.index)))
    with torch.cuda.device(device):
        return _lib.check(fn(*args, torch._C._cuda_getCurrentRawStream(device.index)))


def _workspace(given, need, device):
    """(address, bytes) of the caller's workspace, or of a new one."""
    if given is None:
        given = torch.empty(max(need, 256), dtype=torch.uint8, device=device)
    elif not given.is_cuda or given.device != device or not given.is_contiguous():
        raise ValueError(f"workspace must be a contiguous tensor on {device}")
    return given, given.data_ptr(), given.numel() * given.element_size()


def _on_gpu(t, name, dims):
    if not t.is_cuda:
        raise ValueError(f"{name} must live in GPU memory")
    if t.dim() != dims:
        raise ValueError(f"{name} must have {dims} dimensions, got {t.dim()}")
    return t.device


def _attention_desc(dev, B, n, h, d, scale, h_kv, cap, causal, slopes, doc, prefix):
    h_kv = h if h_kv is None else h_kv
    return AttentionDesc(B, n, h, h_kv, d, int(bool(causal)), scale, cap, _ptr(slopes, "slopes", (h,), torch.float32, dev),
                         _ptr(doc, "doc", (B * n,), torch.int32, dev), _ptr(prefix, "prefix", (B,), torch.int32, dev)), h_kv


def forward_attention_masked(qkv, B, h, d, scale, h_kv=None, cap=0.0, causal=False, slopes=None, doc=None, prefix=None, out=None,
                             lse_out=None):
    """Attention over all tokens of every sample.  qkv [B*n, (h + 2*h_kv)*d] = q | k | v (h_kv None: h).
    cap > 0: scores cap * tanh(score / cap); slopes fp32 [h]: minus slope * distance; causal; prefix int32 [B]: keys before it are
    seen by every query of the sample; doc int32 [B*n]: a token sees its own document only, a negative number is padding.
    Returns (A [B*n, h*d], lse fp32 [B*n, h]); rows that see nothing are +0 with lse -inf."""
    dev = _on_gpu(qkv, "qkv", 2)
    code = _code(qkv)
    rows = qkv.shape[0]
    if B < 1 or rows % B:
        raise ValueError("rows of qkv must be B * n")
    desc, h_kv = _attention_desc(dev, B, rows // B, h, d, scale, h_kv, cap, causal, slopes, doc, prefix)
    p = _ptr(qkv, "qkv", (rows, (h + 2 * h_kv) * d), qkv.dtype, dev)
    if out is None:
        out = torch.empty((rows, h * d), dtype=qkv.dtype, device=dev)
    if lse_out is None:
        lse_out = torch.empty((rows, h), dtype=torch.float32, device=dev)
    _call("sbp_forward_attention_masked", dev, desc, p, code, _ptr(out, "out", (rows, h * d), qkv.dtype, dev),
          _ptr(lse_out, "lse_out", (rows, h), torch.float32, dev))
    return out, lse_out


def backward_attention_masked(qkv_k, A_k, dA_k, lse_k, B, h, d, scale, n=None, idx=None, h_kv=None, cap=0.0, causal=False, slopes=None,
                              doc=None, prefix=None, out=None, workspace=None):
    """Its backward on the kept tokens ("Drop QKV").  qkv_k [B*n_k, (h + 2*h_kv)*d], A_k, dA_k [B*n_k, h*d], lse_k fp32 [B*n_k, h]
    are the kept rows idx (int32 [B*n_k], sample-major; None: all tokens) of the forward's n tokens per sample; doc and prefix as
    in the forward.  Returns dqkv_k [B*n_k, (h + 2*h_kv)*d] (dQ | dK | dV)."""
    dev = _on_gpu(qkv_k, "qkv_k", 2)
    code = _code(qkv_k)
    rows, dt = qkv_k.shape[0], qkv_k.dtype
    if B < 1 or rows % B:
        raise ValueError("rows of qkv_k must be B * n_k")
    n_k = rows // B
    if n is None:
        if idx is not None:
            raise ValueError("n (tokens per sample) is needed with idx")
        n = n_k
    desc, h_kv = _attention_desc(dev, B, n, h, d, scale, h_kv, cap, causal, slopes, doc, prefix)
    width = (h + 2 * h_kv) * d
    p = (_ptr(qkv_k, "qkv_k", (rows, width), dt, dev), _ptr(A_k, "A_k", (rows, h * d), dt, dev), _ptr(dA_k, "dA_k", (rows, h * d), dt, dev),
         _ptr(lse_k, "lse_k", (rows, h), torch.float32, dev), _ptr(idx, "idx", (rows,), torch.int32, dev))
    if out is None:
        out = torch.empty_like(qkv_k)
    po = _ptr(out, "out", (rows, width), dt, dev)
    workspace, pw, nw = _workspace(workspace, _lib.lib().sbp_backward_attention_masked_workspace(desc, n_k, code), dev)
    _call("sbp_backward_attention_masked", dev, desc, *p, n_k, code, po, pw, nw)
    return out


def _norm_desc(dev, M, C, gate, alpha, gamma_post, beta_post, gamma_pre, beta_pre, kind, eps):
    f32, G = torch.float32, 1
    if gate is not None:
        if gate.dim() == 1:
            gate = gate.unsqueeze(0)
        G = gate.shape[0]
    return ResidualNormDesc(M, C, kind, G, alpha, eps, 0, _ptr(gate, "gate", (G, C), f32, dev), _ptr(gamma_post, "gamma_post", (C,), f32, dev),
                            _ptr(beta_post, "beta_post", (C,), f32, dev), _ptr(gamma_pre, "gamma_pre", (C,), f32, dev),
                            _ptr(beta_pre, "beta_pre", (C,), f32, dev)), G


def forward_residual_norm(x, y=None, gate=None, alpha=1.0, gamma_post=None, beta_post=None, gamma_pre=None, beta_pre=None, kind=NORM_RMS,
                          eps=1e-5, x_out=None, z=None):
    """x_out = alpha * x + gate * post(y), z = pre(x_out): the norm after a block, its gate, the residual sum and the next block's norm.
    x, y [M, C]; gate fp32 [C] or [G, C] (row r has gate[r // (M / G)]); gammas, betas fp32 [C], gamma None: that norm is left out.
    Returns (x_out, z); z is None without gamma_pre.  x_out may be x (in place)."""
    dev = _on_gpu(x, "x", 2)
    code = _code(x)
    M, C = x.shape
    desc, _ = _norm_desc(dev, M, C, gate, alpha, gamma_post, beta_post, gamma_pre, beta_pre, kind, eps)
    px, py = _ptr(x, "x", (M, C), x.dtype, dev), _ptr(y, "y", (M, C), x.dtype, dev)
    if x_out is None:
        x_out = torch.empty_like(x)
    if z is None and gamma_pre is not None:
        z = torch.empty_like(x)
    _call("sbp_forward_residual_norm", dev, desc, px, py, code, _ptr(x_out, "x_out", (M, C), x.dtype, dev), _ptr(z, "z", (M, C), x.dtype, dev))
    return x_out, z


_PARAM_GRADS = ("dgate", "dgamma_post", "dbeta_post", "dgamma_pre", "dbeta_pre")


def backward_residual_norm(dx_out, dz_k, x_out_k, y_k, idx, M, gate=None, alpha=1.0, gamma_post=None, beta_post=None, gamma_pre=None,
                           kind=NORM_RMS, eps=1e-5, inv=None, flags=0, want=None, dx=None, dy_k=None, grads=None, workspace=None):
    """Backward of forward_residual_norm on the kept rows idx.  dx_out [M, C] (the residual stream's gradient; None: 0), dz_k, x_out_k,
    y_k [K, C].  Returns a dict with the entries named in `want`: dx [M, C] (alpha * dx_out in the dropped rows), dy_k [K, C], and fp32
    dgate, dgamma_post, dbeta_post, dgamma_pre, dbeta_pre; by default dx, dy_k and the gradient of every vector given.
    FLAG_DX_COMPACT: dx_out and dx are [K, C].  `grads`: preallocated parameter gradients by name (needed with FLAG_ACCUMULATE_DW)."""
    some = next((t for t in (y_k, dz_k, dx_out) if t is not None), None)
    if some is None:
        raise ValueError("one of dx_out, dz_k and y_k is needed")
    dev = _on_gpu(some, "dx_out, dz_k or y_k", 2)
    code, dt, C = _code(some), some.dtype, some.shape[1]
    f32 = torch.float32
    compact = bool(flags & _FLAG_DX_COMPACT)
    kept = y_k if y_k is not None else dz_k
    K = idx.numel() if idx is not None else kept.shape[0] if kept is not None else dx_out.shape[0]
    desc, G = _norm_desc(dev, M, C, gate, alpha, gamma_post, beta_post, gamma_pre, None, kind, eps)
    if want is None:
        want = ["dx", "dy_k"] + ["dgate"] * (gate is not None) + ["dgamma_post"] * (gamma_post is not None)
        want += ["dbeta_post"] * (beta_post is not None) + ["dgamma_pre"] * (dz_k is not None)
    for name in want:
        if name not in ("dx", "dy_k", *_PARAM_GRADS):
            raise ValueError(f"unknown output {name}")
    rows = K if compact else M
    p = (_ptr(dx_out, "dx_out", (rows, C), dt, dev), _ptr(dz_k, "dz_k", (K, C), dt, dev), _ptr(x_out_k, "x_out_k", (K, C), dt, dev),
         _ptr(y_k, "y_k", (K, C), dt, dev), _ptr(idx, "idx", (K,), torch.int32, dev), _ptr(inv, "inv", (M,), torch.int32, dev))
    out = {}
    if "dx" in want:
        out["dx"] = torch.empty((rows, C), dtype=dt, device=dev) if dx is None else dx
    if "dy_k" in want:
        out["dy_k"] = torch.empty((K, C), dtype=dt, device=dev) if dy_k is None else dy_k
    for name in _PARAM_GRADS:
        if name in want:
            given = (grads or {}).get(name)
            if given is None and flags & _FLAG_ACCUMULATE:
                raise ValueError(f"{name} has to be given in grads to be accumulated into")
            out[name] = torch.empty(gate.shape if name == "dgate" else (C,), dtype=f32, device=dev) if given is None else given
    g = ResidualNormGrads(*[_ptr(out.get(name), name, gate.shape if name == "dgate" and gate is not None else (C,), f32, dev)
                            for name in _PARAM_GRADS])
    px, py = _ptr(out.get("dx"), "dx", (rows, C), dt, dev), _ptr(out.get("dy_k"), "dy_k", (K, C), dt, dev)
    workspace, pw, nw = _workspace(workspace, _lib.lib().sbp_backward_residual_norm_workspace(desc, K, code, flags), dev)
    _call("sbp_backward_residual_norm", dev, desc, *p, K, code, px, py, g, pw, nw, flags)
    return out


def _tokens(tokens, dev):
    if tokens.dtype not in (torch.int32, torch.int64):
        raise TypeError(f"tokens must be int32 or int64, got {tokens.dtype}")
    return _ptr(tokens, "tokens", tokens.shape, tokens.dtype, dev), tokens.element_size()


def forward_embedding(tokens, table, scale=1.0, out=None):
    """E[r] = scale * table[tokens[r]]: [*tokens.shape, C]; tokens int32 or int64, one outside the table gives a row of +0."""
    dev = _on_gpu(table, "table", 2)
    code = _code(table)
    V, C = table.shape
    pt, size = _tokens(tokens, dev)
    p = _ptr(table, "table", (V, C), table.dtype, dev)
    shape = (*tokens.shape, C)
    if out is None:
        out = torch.empty(shape, dtype=table.dtype, device=dev)
    _call("sbp_forward_embedding", dev, pt, size, p, tokens.numel(), V, C, scale, code, _ptr(out, "out", shape, table.dtype, dev))
    return out


def backward_embedding(dE, tokens, V, idx=None, scale=1.0, flags=0, dtable=None, workspace=None):
    """dtable [V, C] fp32 (bf16 with FLAG_DW_OUT_BF16) from the kept rows idx (int32 [K]; None: all): scale * the sum of the rows of dE
    whose token it is, +0 elsewhere.  dE [M, C], or [K, C] with FLAG_DY_COMPACT; tokens [M] int32 or int64.  FLAG_ACCUMULATE_DW adds to
    the given dtable and touches no other row."""
    dev = _on_gpu(dE, "dE", 2)
    code = _code(dE)
    M, C = tokens.numel(), dE.shape[1]
    K = M if idx is None else idx.numel()
    pt, size = _tokens(tokens, dev)
    p = _ptr(dE, "dE", (K if flags & _FLAG_DY_COMPACT else M, C), dE.dtype, dev)
    pi = _ptr(idx, "idx", (K,), torch.int32, dev)
    dt = torch.bfloat16 if flags & _FLAG_OUT_BF16 else torch.float32
    if dtable is None:
        if flags & _FLAG_ACCUMULATE:
            raise ValueError("dtable has to be given to be accumulated into")
        dtable = torch.empty((V, C), dtype=dt, device=dev)
    po = _ptr(dtable, "dtable", (V, C), dt, dev)
    workspace, pw, nw = _workspace(workspace, _lib.lib().sbp_backward_embedding_workspace(M, K, V, C, code, flags), dev)
    _call("sbp_backward_embedding", dev, p, pt, size, pi, M, K, V, C, scale, code, po, pw, nw, flags)
    return dtable
