"""Plain CPU oracle of the language-model steps: masked attention, the norms between blocks, the token table.

TEST INFRASTRUCTURE.  fp64 write-out of the definitions in include/sbp_lm.h, sharing no code with the HIP kernels.  Arrays hold
one sample where the definition is per sample: q [n, h, d], k and v [n, h_kv, d], positions and documents [n].
"""
from __future__ import annotations

import numpy as np

NORM_RMS, NORM_LAYER = 0, 1


def visible(pos, doc=None, causal=False, prefix=0):
    """[n, n] truth values: query i sees key j."""
    pos = np.asarray(pos, dtype=np.int64)
    n = pos.size
    see = np.ones((n, n), dtype=bool)
    for i in range(n):
        if causal:
            see[i] &= (pos <= pos[i]) | (pos < prefix)
        if doc is not None:
            see[i] &= (np.asarray(doc) == doc[i]) & (doc[i] >= 0)
    return see


def scores(q, k, pos, scale, cap=0.0, slope=0.0):
    """Scores of one head and the derivative of the cap."""
    z = scale * (q @ k.T)
    t = np.tanh(z / cap) if cap else np.zeros_like(z)
    s = cap * t if cap else z
    pos = np.asarray(pos, dtype=np.float64)
    return s - slope * np.abs(pos[:, None] - pos[None, :]), 1.0 - t * t


def attention(q, k, v, pos, scale, cap=0.0, slopes=None, doc=None, causal=False, prefix=0):
    """(A [n, h, d], lse [n, h]) over all tokens given."""
    n, h, d = q.shape
    group = h // k.shape[1]
    see = visible(pos, doc, causal, prefix)
    A, lse = np.zeros((n, h, d)), np.full((n, h), -np.inf)
    for a in range(h):
        s, _ = scores(q[:, a], k[:, a // group], pos, scale, cap, 0.0 if slopes is None else slopes[a])
        for i in range(n):
            on = see[i]
            if not on.any():
                continue
            m = s[i, on].max()
            e = np.exp(s[i, on] - m)
            lse[i, a] = m + np.log(e.sum())
            A[i, a] = (e / e.sum()) @ v[on, a // group]
    return A, lse


def attention_backward(q, k, v, A, dA, lse, pos, scale, cap=0.0, slopes=None, doc=None, causal=False, prefix=0):
    """(dq, dk, dv) over the kept tokens given (lse, A of the forward over all of them)."""
    n, h, d = q.shape
    group = h // k.shape[1]
    see = visible(pos, doc, causal, prefix)
    dq, dk, dv = np.zeros(q.shape), np.zeros(k.shape), np.zeros(v.shape)
    for a in range(h):
        c = a // group
        s, slope = scores(q[:, a], k[:, c], pos, scale, cap, 0.0 if slopes is None else slopes[a])
        for i in range(n):
            on = see[i]
            if not on.any():
                continue
            p = np.exp(s[i, on] - lse[i, a])
            dm = p * (v[on, c] @ dA[i, a] - dA[i, a] @ A[i, a]) * slope[i, on] * scale
            dq[i, a] = dm @ k[on, c]
            dk[on, c] += dm[:, None] * q[i, a]
            dv[on, c] += p[:, None] * dA[i, a]
    return dq, dk, dv


def norm_rows(x, kind, eps):
    """(normalised rows, 1 / deviation [M, 1])."""
    if kind == NORM_LAYER:
        x = x - x.mean(axis=1, keepdims=True)
    r = 1.0 / np.sqrt((x * x).mean(axis=1, keepdims=True) + eps)
    return x * r, r


def norm_backward(g, hat, r, kind):
    out = g - hat * (g * hat).mean(axis=1, keepdims=True)
    if kind == NORM_LAYER:
        out = out - g.mean(axis=1, keepdims=True)
    return out * r


def _spread(gate, rows):
    return np.repeat(gate, rows // gate.shape[0], axis=0)


def residual_norm(x, y, kind, eps, alpha=1.0, gate=None, gamma_post=None, beta_post=None, gamma_pre=None, beta_pre=None):
    """(x_out, z)."""
    out = alpha * x
    if y is not None:
        u = y
        if gamma_post is not None:
            u = norm_rows(y, kind, eps)[0] * gamma_post + (0.0 if beta_post is None else beta_post)
        out = out + (u if gate is None else u * _spread(gate, x.shape[0]))
    z = None
    if gamma_pre is not None:
        z = norm_rows(out, kind, eps)[0] * gamma_pre + (0.0 if beta_pre is None else beta_pre)
    return out, z


def residual_norm_backward(dx_out, dz, x_out, y, idx, M, kind, eps, alpha=1.0, gate=None, gamma_post=None, beta_post=None, gamma_pre=None):
    """Dict of dx [M, C], dy [K, C] and the parameter gradients; dx_out [M, C], the others [K, C].  "terms": for the rows of dx (kept ones)
    and dy the largest of the terms whose sum they are, which may cancel (to nothing for one channel without a mean)."""
    C = (y if y is not None else dz).shape[1]
    K = len(idx)
    dx_out = np.zeros((M, C)) if dx_out is None else dx_out
    t = dx_out[idx].copy()
    out = {}
    terms = np.abs(t).max(axis=1, keepdims=True)
    if dz is not None:
        hat, r = norm_rows(x_out, kind, eps)
        terms = terms + r * np.abs(dz * gamma_pre).max(axis=1, keepdims=True) * np.abs(hat).max(axis=1, keepdims=True).clip(1.0)
        t += norm_backward(dz * gamma_pre, hat, r, kind)
        out["dgamma_pre"], out["dbeta_pre"] = (dz * hat).sum(axis=0), dz.sum(axis=0)
    dx = alpha * dx_out
    dx[idx] = alpha * t
    out["dx"] = dx
    du = t if gate is None else t * _spread(gate, K)
    out["dy_k"] = du
    out["terms"] = {"dx": np.zeros((M, 1)), "dy_k": terms * (1.0 if gate is None else np.abs(_spread(gate, K)).max(axis=1, keepdims=True))}
    out["terms"]["dx"][idx] = abs(alpha) * terms
    if y is not None:
        hat, r = norm_rows(y, kind, eps) if gamma_post is not None else (y, None)
        u = hat if gamma_post is None else hat * gamma_post + (0.0 if beta_post is None else beta_post)
        if gate is not None:
            out["dgate"] = (t * u).reshape(gate.shape[0], K // gate.shape[0], C).sum(axis=1)
        if gamma_post is not None:
            out["dgamma_post"], out["dbeta_post"] = (du * hat).sum(axis=0), du.sum(axis=0)
            out["dy_k"] = norm_backward(du * gamma_post, hat, r, kind)
            out["terms"]["dy_k"] = out["terms"]["dy_k"] * r * np.abs(gamma_post).max() * np.abs(hat).max(axis=1, keepdims=True).clip(1.0)
    return out


def embedding(tokens, table, scale):
    E = np.zeros((len(tokens), table.shape[1]))
    for r, tok in enumerate(tokens):
        if 0 <= tok < table.shape[0]:
            E[r] = scale * table[tok]
    return E


def embedding_backward(dE_k, tokens_k, V, scale):
    out = np.zeros((V, dE_k.shape[1]))
    for row, tok in zip(dE_k, tokens_k):
        if 0 <= tok < V:
            out[tok] += scale * row
    return out
