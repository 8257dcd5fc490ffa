"""The language-model steps in bf16 as they are used together, every call held to its definition in 64 bits on the inputs that it had: a chain of
roundings to bf16 is bounded call by call, where a bound of the whole chain would be as wide as its results."""
import math

import numpy as np
import pytest
import torch

import paper_2210_00129_amd as sbp
from lm_attention_gpu import Long
from lm_bounds import EPS, NORM_LAYER, NORM_RMS, Near, f32, norm, number, statistics

pytestmark = pytest.mark.gpu
STEP = 2.0 ** -8               # a rounding to bf16
U = 2.0 ** -24
BF16 = torch.bfloat16


def _held(got, ref, err, what, step=STEP):
    over = (got.double() - ref).abs() - (1.01 * (err + step * (ref.abs() + err)) + 1e-30)
    assert torch.isfinite(got).all() and float(over.max()) <= 0, (what, float(over.max()))


def _near(t):
    return Near(t.double().reshape(1, -1) if t.dim() == 1 else t.double())


def _product(got, a, b, what, step):
    """got = a b, sums in fp32 over the inner dimension."""
    a, b = a.double(), b.double().contiguous()
    _held(got, a @ b, (a.shape[1] + 8) * U * (a.abs() @ b.abs()), what, step)


@pytest.mark.parametrize("B,N,V,H,HK,D,C,k", [(2, 40, 50, 4, 2, 16, 64, 2), (3, 196, 400, 4, 1, 64, 264, 1), (1, 512, 1000, 2, 2, 128, 512, 3)])
@pytest.mark.parametrize("kind", [NORM_RMS, NORM_LAYER])
def test_every_call_of_a_step(B, N, V, H, HK, D, C, k, kind):
    g, M, width = torch.Generator(device="cuda").manual_seed(50), B * N, (H + 2 * HK) * D

    def rand(*s, by=1.0, at=0.0):
        return at + by * torch.randn(*s, generator=g, device="cuda")
    scale, alpha = math.sqrt(C), 0.75
    table, Wqkv, Wo = (t.to(BF16) for t in (rand(V, C, by=1 / scale), rand(width, C, by=C ** -0.5), rand(C, H * D, by=(H * D) ** -0.5)))
    g0, b0, gate, gp, bp, gn, bn = rand(C, by=0.1, at=1), rand(C, by=0.1), rand(B, C), rand(C, by=0.1, at=1), rand(C, by=0.1), rand(C, by=0.1, at=1), rand(C, by=0.1)
    dx1, dz1 = rand(M, C).to(BF16), rand(M, C).to(BF16)
    tokens = torch.randint(0, V, (M,), generator=g, device="cuda")
    doc = torch.from_numpy(np.sort(np.random.default_rng(1).integers(0, 3, size=(B, N)), axis=1).astype(np.int32).reshape(-1)).cuda()
    slopes = torch.tensor([0.5 / (i + 1) for i in range(H)], device="cuda")
    attn = dict(B=B, h=H, d=D, scale=D ** -0.5, h_kv=HK, cap=8.0, causal=True, slopes=slopes, doc=doc)

    # forward
    x0 = sbp.forward_embedding(tokens, table, scale)
    _held(x0, table.double()[tokens] * f32(scale), U * table.double()[tokens].abs() * scale, "lookup")
    x0_again, z0 = sbp.forward_residual_norm(x0, gamma_pre=g0, beta_pre=b0, kind=kind, eps=EPS)
    assert torch.equal(x0_again, x0)
    r = norm(_near(x0), _near(g0), _near(b0), kind)
    _held(z0, r.v, r.e, "z0")
    qkv = z0 @ Wqkv.T
    A, lse = sbp.forward_attention_masked(qkv, **attn)
    y = A @ Wo.T
    step = dict(gate=gate, alpha=alpha, gamma_post=gp, beta_post=bp, gamma_pre=gn, kind=kind, eps=EPS)
    x1, z1 = sbp.forward_residual_norm(x0, y, beta_pre=bn, **step)
    gates = Near(gate.double().repeat_interleave(N, 0))
    r = _near(x0) * number(alpha, x0) + norm(_near(y), _near(gp), _near(bp), kind) * gates
    _held(x1, r.v, r.e, "x1")
    r = norm(r, _near(gn), _near(bn), kind)
    _held(z1, r.v, r.e, "z1")

    # backward on a drawn keep-set
    idx, inv = sbp.sample_indices(B, 0, N, 1, k, seed=9, stream_id=0, mode=sbp.TEMPORAL, cell=4, want_inv=True)
    at, K = idx.long(), idx.numel()
    x0_k, z0_k, qkv_k, A_k, y_k, x1_k, dz1_k = (sbp.forward_cache(t, idx) for t in (x0, z0, qkv, A, y, x1, dz1))
    for part, whole in ((x0_k, x0), (z0_k, z0), (qkv_k, qkv), (A_k, A), (y_k, y), (x1_k, x1), (dz1_k, dz1)):
        assert torch.equal(part, whole[at])
    lse_k = lse[at].contiguous()
    got = sbp.backward_residual_norm(dx1, dz1_k, x1_k, y_k, idx, M, inv=inv, **step,
                                     want=("dx", "dy_k", "dgate", "dgamma_post", "dbeta_post", "dgamma_pre", "dbeta_pre"))

    def through(g_out, x, gamma):
        """The gradient through a norm of x: (of x, of gamma's terms, the normalised rows)."""
        c, r = statistics(_near(x), kind)
        h, hat = g_out * _near(gamma), c * r
        into = h - hat * (h * hat).mean()
        return r * (into - h.mean() if kind == NORM_LAYER else into), g_out * hat, hat
    gates_k = Near(gate.double().repeat_interleave(K // B, 0))
    into, hats, _ = through(_near(dz1_k), x1_k, gn)
    t = _near(dx1[at]) + into
    r = number(alpha, x0) * t
    _held(got["dx"][at], r.v, r.e, "dx")
    u = t * gates_k
    r, post, hat = through(u, y_k, gp)
    _held(got["dy_k"], r.v, r.e, "dy_k")

    def total(n):
        return n.total(0, K + 40)
    for name, ref in (("dgamma_pre", total(hats)), ("dbeta_pre", total(_near(dz1_k))), ("dgamma_post", total(post)), ("dbeta_post", total(u))):
        _held(got[name].reshape(1, -1), ref.v, ref.e, name, 0.0)
    s = t * (hat * _near(gp) + _near(bp))
    per = [Near(s.v[b * (K // B):(b + 1) * (K // B)], s.e[b * (K // B):(b + 1) * (K // B)]).total(0, K + 40) for b in range(B)]
    # (the kernel sums t hat and t by themselves: their errors are those of the sums' absolute terms)
    slack = (K + 60) * U * ((t * hat).v.abs() * gp.abs().double() + t.v.abs() * bp.abs().double()).view(B, K // B, C).sum(1)
    _held(got["dgate"], torch.cat([p.v for p in per]), torch.cat([p.e for p in per]) + slack, "dgate", 0.0)

    both = sbp.FLAG_DY_COMPACT | sbp.FLAG_DX_COMPACT
    dWo, _, dA_k = sbp.backward_linear(got["dy_k"], idx, A_k, Wo, M=M, flags=both, want=("dW", "dX"))
    _product(dWo, got["dy_k"].t(), A_k, "dWo", 0.0)
    _product(dA_k, got["dy_k"], Wo, "dA", STEP)
    dqkv_k = sbp.backward_attention_masked(qkv_k, A_k, dA_k, lse_k, n=N, idx=idx, **attn)
    for b in range(B):
        rows, kept = slice(b * N, (b + 1) * N), slice(b * (K // B), (b + 1) * (K // B))
        c = Long(N, H, HK, D, "bf16", cap=8.0, causal=True, doc=doc[rows], scale=D ** -0.5, kept=at[kept] - b * N)
        c.slopes, c.qkv = slopes, qkv[rows]
        c.hold_forward(A[rows], lse[rows])
        c.hold_backward(*(t[kept] for t in (qkv_k, A_k, dA_k, lse_k, dqkv_k)))
    dWqkv, _, dz0_k = sbp.backward_linear(dqkv_k, idx, z0_k, Wqkv, M=M, flags=both, want=("dW", "dX"))
    _product(dWqkv, dqkv_k.t(), z0_k, "dWqkv", 0.0)
    _product(dz0_k, dqkv_k, Wqkv, "dz0", STEP)
    first = sbp.backward_residual_norm(got["dx"], dz0_k, x0_k, None, idx, M, inv=inv, gamma_pre=g0, kind=kind, eps=EPS, want=("dx", "dgamma_pre", "dbeta_pre"))
    into, hats, _ = through(_near(dz0_k), x0_k, g0)
    r = _near(got["dx"][at]) + into
    _held(first["dx"][at], r.v, r.e, "first dx")
    for name, ref in (("dgamma_pre", total(hats)), ("dbeta_pre", total(_near(dz0_k)))):
        _held(first[name].reshape(1, -1), ref.v, ref.e, "first " + name, 0.0)
    dropped = inv < 0
    assert torch.equal(first["dx"][dropped], got["dx"][dropped])
    dtable = sbp.backward_embedding(first["dx"], tokens, V, idx=idx, scale=scale)
    ref, size = (torch.zeros(V, C, dtype=torch.float64, device="cuda") for _ in range(2))
    ref.index_add_(0, tokens[at], first["dx"].double()[at] * f32(scale))
    size.index_add_(0, tokens[at], first["dx"].double()[at].abs() * f32(scale))
    _held(dtable, ref, (K + 4) * U * size, "dtable", 0.0)
