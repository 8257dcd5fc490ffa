"""The oracle of the language-model steps against automatic differentiation in fp64 and against differences (CPU only)."""
import math

import numpy as np
import pytest
import torch

from oracle import lm_oracle as lm

EPS = 1e-5


def _attention_torch(q, k, v, pos, scale, cap, slopes, doc, causal, prefix):
    """The forward's definition in differentiable operations: q [n, h, d], k, v [n, hk, d]; every row has to see something."""
    n, h, d = q.shape
    rep = h // k.shape[1]
    k, v = k.repeat_interleave(rep, 1), v.repeat_interleave(rep, 1)
    s = torch.einsum("ihd,jhd->hij", q, k) * scale
    if cap:
        s = cap * torch.tanh(s / cap)
    t = torch.as_tensor(pos)
    if slopes is not None:
        s = s - torch.as_tensor(slopes, dtype=torch.float64)[:, None, None] * (t[:, None] - t[None]).abs()
    see = torch.ones(n, n, dtype=torch.bool)
    if causal:
        see = (t[None] <= t[:, None]) | (t[None] < prefix)
    if doc is not None:
        see = see & (torch.as_tensor(doc)[:, None] == torch.as_tensor(doc)[None])
    s = s.masked_fill(~see, -math.inf)
    return torch.einsum("hij,jhd->ihd", torch.softmax(s, 2), v), torch.logsumexp(s, 2).t()


@pytest.mark.parametrize("cap,bias,docs,causal,prefix,hk", [(0, False, False, False, 0, 2), (3.0, False, False, True, 0, 1), (0, True, True, True, 4, 2),
                                                            (2.0, True, True, False, 0, 1), (1.5, True, False, True, 5, 2)])
def test_attention_and_its_gradients(cap, bias, docs, causal, prefix, hk):
    g = torch.Generator().manual_seed(3)
    n, h, d = 11, 2, 4
    q = torch.randn(n, h, d, generator=g, dtype=torch.float64, requires_grad=True)
    k, v = (torch.randn(n, hk, d, generator=g, dtype=torch.float64, requires_grad=True) for _ in range(2))
    dA = torch.randn(n, h, d, generator=g, dtype=torch.float64)
    pos = np.array([3, 0, 7, 1, 2, 9, 4, 5, 6, 8, 10])                       # any order of positions
    slopes = [0.3, 0.05] if bias else None
    doc = np.array([0, 0, 1, 0, 1, 2, 1, 1, 2, 2, 2]) if docs else None
    A, lse = _attention_torch(q, k, v, pos, 0.5, cap, slopes, doc, causal, prefix)
    wq, wk, wv = torch.autograd.grad(A, (q, k, v), dA)
    x = [t.detach().numpy() for t in (q, k, v)]
    kw = dict(cap=cap, slopes=slopes, doc=doc, causal=causal, prefix=prefix)
    oA, ol = lm.attention(*x, pos, 0.5, **kw)
    assert np.allclose(oA, A.detach().numpy(), atol=1e-12) and np.allclose(ol, lse.detach().numpy(), atol=1e-12)
    got = lm.attention_backward(*x, oA, dA.numpy(), ol, pos, 0.5, **kw)
    for a, b in zip(got, (wq, wk, wv)):
        assert np.allclose(a, b.numpy(), atol=1e-12)


def test_attention_gradient_against_differences():
    rng = np.random.default_rng(0)
    n, h, d = 7, 2, 4
    q, k, v, dA = rng.standard_normal((n, h, d)), rng.standard_normal((n, 1, d)), rng.standard_normal((n, 1, d)), rng.standard_normal((n, h, d))
    kw = dict(cap=2.0, slopes=[0.2, 0.1], doc=np.array([0, 0, 0, 1, 1, 1, -1]), causal=True, prefix=2)
    A, lse = lm.attention(q, k, v, np.arange(n), 0.6, **kw)
    assert np.all(A[6] == 0) and np.all(lse[6] == -np.inf)
    got = lm.attention_backward(q, k, v, A, dA, lse, np.arange(n), 0.6, **kw)
    x = [q, k, v]
    for which in range(3):
        for at in [(0, 0, 1), (2, 0, 3), (4, 0, 0), (6, 0, 2)]:
            f = []
            for e in (1e-5, -1e-5):
                y = [t.copy() for t in x]
                y[which][at] += e
                f.append((lm.attention(*y, np.arange(n), 0.6, **kw)[0] * dA).sum())
            assert abs((f[0] - f[1]) / 2e-5 - got[which][at]) < 1e-8


def test_dropped_tokens_take_no_part():
    """The kept backward is the full one with dM set to zero where the query or the key is dropped."""
    rng = np.random.default_rng(1)
    n, d = 9, 4
    q, k, v, dA = (rng.standard_normal((n, 1, d)) for _ in range(4))
    pos = np.arange(n)
    A, lse = lm.attention(q, k, v, pos, 0.5, causal=True)
    keep = np.array([1, 2, 5, 8])
    got = lm.attention_backward(q[keep], k[keep], v[keep], A[keep], dA[keep], lse[keep], keep, 0.5, causal=True)
    s, _ = lm.scores(q[:, 0], k[:, 0], pos, 0.5)
    P = np.where(lm.visible(pos, causal=True), np.exp(s - lse), 0.0)
    dM = P * (dA[:, 0] @ v[:, 0].T - (dA[:, 0] * A[:, 0]).sum(1, keepdims=True))
    on = np.isin(pos, keep)
    dM, P = np.where(on[:, None] & on[None], dM, 0.0), np.where(on[:, None] & on[None], P, 0.0)
    assert np.allclose(got[0][:, 0], 0.5 * (dM @ k[:, 0])[keep]) and np.allclose(got[1][:, 0], 0.5 * (dM.T @ q[:, 0])[keep])
    assert np.allclose(got[2][:, 0], (P.T @ dA[:, 0])[keep])


@pytest.mark.parametrize("kind", [lm.NORM_RMS, lm.NORM_LAYER])
@pytest.mark.parametrize("post,pre,beta,G", [(True, True, True, 1), (True, True, False, 3), (False, True, True, 2), (True, False, True, 0)])
def test_residual_norm_gradients(kind, post, pre, beta, G):
    g = torch.Generator().manual_seed(5)
    M, C = 12, 7

    def leaf(on, *shape):
        return torch.randn(*shape, generator=g, dtype=torch.float64, requires_grad=True) if on else None

    x, y = leaf(True, M, C), leaf(True, M, C)
    gate, gp, bp, gn, bn = leaf(G, G, C), leaf(post, C), leaf(post and beta, C), leaf(pre, C), leaf(pre and beta, C)

    def norm(t):
        if kind == lm.NORM_LAYER:
            t = t - t.mean(1, keepdim=True)
        return t / torch.sqrt((t * t).mean(1, keepdim=True) + EPS)

    def zero(t):
        return 0.0 if t is None else t

    u = norm(y) * gp + zero(bp) if post else y
    x_out = 0.7 * x + (u * gate.repeat_interleave(M // G, 0) if G else u)
    z = norm(x_out) * gn + zero(bn) if pre else None
    d_out, dz = torch.randn(M, C, generator=g, dtype=torch.float64), torch.randn(M, C, generator=g, dtype=torch.float64)
    leaves = dict(dx=x, dy_k=y, dgate=gate, dgamma_post=gp, dbeta_post=bp, dgamma_pre=gn, dbeta_pre=bn)
    leaves = {k: t for k, t in leaves.items() if t is not None}
    want = torch.autograd.grad((x_out * d_out).sum() + ((z * dz).sum() if pre else 0.0), list(leaves.values()))

    def num(t):
        return None if t is None else t.detach().numpy()

    kw = dict(alpha=0.7, gate=num(gate), gamma_post=num(gp), beta_post=num(bp), gamma_pre=num(gn))
    ox, oz = lm.residual_norm(num(x), num(y), kind, EPS, beta_pre=num(bn), **kw)
    assert np.allclose(ox, num(x_out)) and (oz is None) == (z is None) and (z is None or np.allclose(oz, num(z)))
    got = lm.residual_norm_backward(d_out.numpy(), dz.numpy() if pre else None, num(x_out), num(y), np.arange(M), M, kind, EPS, **kw)
    for name, w in zip(leaves, want):
        assert np.allclose(got[name], w.numpy(), atol=1e-11), name


def test_residual_norm_dropped_rows_pass_the_stream_through():
    rng = np.random.default_rng(2)
    d_out, dz, x, y = rng.standard_normal((6, 5)), *(rng.standard_normal((2, 5)) for _ in range(3))
    got = lm.residual_norm_backward(d_out, dz, x, y, np.array([1, 4]), 6, 0, EPS, alpha=0.5, gamma_post=np.ones(5), gamma_pre=np.ones(5))
    assert np.allclose(got["dx"][[0, 2, 3, 5]], 0.5 * d_out[[0, 2, 3, 5]])


def test_embedding_gradient():
    rng = np.random.default_rng(4)
    tokens = np.array([3, 0, 3, -1, 7, 2, 3])
    table = rng.standard_normal((5, 3))
    E = lm.embedding(tokens, table, 2.0)
    assert np.all(E[[3, 4]] == 0) and np.allclose(E[2], 2.0 * table[3])
    dE = rng.standard_normal((7, 3))
    t = torch.tensor(table, requires_grad=True)
    ok = [0, 1, 2, 5, 6]
    (2.0 * t[torch.tensor(tokens[ok])] * torch.tensor(dE[ok])).sum().backward()
    assert np.allclose(lm.embedding_backward(dE, tokens, 5, 2.0), t.grad.numpy())
