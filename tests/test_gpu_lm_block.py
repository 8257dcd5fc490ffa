"""The language-model steps as they are used together: token table, norm, projection to q, k and v, masked attention, output projection,
residual sum with both norms, and SBP's backward through all of it, on drawn keep-sets and with every token kept."""
import math

import numpy as np
import pytest
import torch

import paper_2210_00129_amd as sbp
from oracle import lm_oracle as lm

pytestmark = pytest.mark.gpu

B, N, V, H, HK, D = 2, 40, 50, 4, 2, 16
C, M = H * D, 2 * 40
QKV = (H + 2 * HK) * D
ALPHA, SCALE, EPS, CAP = 0.75, math.sqrt(C), 1e-5, 8.0
KIND = sbp.NORM_LAYER

# Every step adds up at most T = 3 C terms in fp32, each sum off by at most T 2^-24 of the sum of its absolute terms, which for random
# signs is sqrt(T) times its result; 2 x 7 steps lie one behind the other, and the norms and the softmax scale errors by factors around 1.
TOLERANCE = 14 * (3 * C) * math.sqrt(3 * C) * 2.0 ** -24


def _model(seed):
    g = torch.Generator().manual_seed(seed)

    def rand(*s, by=1.0):
        return by * torch.randn(*s, generator=g)
    p = dict(table=rand(V, C, by=1 / SCALE), g0=1 + rand(C, by=0.1), b0=rand(C, by=0.1), Wqkv=rand(QKV, C, by=C ** -0.5), Wo=rand(C, C, by=C ** -0.5),
             gate=rand(B, C), gp=1 + rand(C, by=0.1), bp=rand(C, by=0.1), gn=1 + rand(C, by=0.1), bn=rand(C, by=0.1))
    tokens = torch.randint(0, V, (M,), generator=g)
    doc = torch.from_numpy(np.sort(np.random.default_rng(seed).integers(0, 3, size=(B, N)), axis=1).astype(np.int32).reshape(-1))
    slopes = torch.tensor([0.5, 0.25, 0.125, 0.0625])
    return p, tokens, doc, slopes, rand(M, C), rand(M, C)                 # and the gradients of both outputs


def _run(p, tokens, doc, slopes, dx1, dz1, idx):
    """Forward, then the backward on the kept rows idx; every result of it."""
    attn = dict(B=B, h=H, d=D, scale=D ** -0.5, h_kv=HK, cap=CAP, causal=True, slopes=slopes, doc=doc)
    x0 = sbp.forward_embedding(tokens, p["table"], SCALE)
    _, z0 = sbp.forward_residual_norm(x0, gamma_pre=p["g0"], beta_pre=p["b0"], kind=KIND, eps=EPS)
    qkv = z0 @ p["Wqkv"].T
    A, lse = sbp.forward_attention_masked(qkv, **attn)
    y = A @ p["Wo"].T
    step = dict(gate=p["gate"], alpha=ALPHA, gamma_post=p["gp"], beta_post=p["bp"], gamma_pre=p["gn"], kind=KIND, eps=EPS)
    x1, z1 = sbp.forward_residual_norm(x0, y, beta_pre=p["bn"], **step)
    # what a layer keeps
    x0_k, z0_k, qkv_k, A_k, y_k, x1_k, dz1_k = (sbp.forward_cache(t, idx) for t in (x0, z0, qkv, A, y, x1, dz1))
    lse_k = lse[idx.long()].contiguous()
    g = sbp.backward_residual_norm(dx1, dz1_k, x1_k, y_k, idx, M, **step, want=("dx", "dy_k", "dgate", "dgamma_post", "dbeta_post", "dgamma_pre", "dbeta_pre"))
    both = sbp.FLAG_DY_COMPACT | sbp.FLAG_DX_COMPACT
    dWo, _, dA_k = sbp.backward_linear(g["dy_k"], idx, A_k, p["Wo"], M=M, flags=both, want=("dW", "dX"))
    dqkv_k = sbp.backward_attention_masked(qkv_k, A_k, dA_k, lse_k, n=N, idx=idx, **attn)
    dWqkv, _, dz0_k = sbp.backward_linear(dqkv_k, idx, z0_k, p["Wqkv"], M=M, flags=both, want=("dW", "dX"))
    g0 = sbp.backward_residual_norm(g["dx"], dz0_k, x0_k, None, idx, M, gamma_pre=p["g0"], kind=KIND, eps=EPS, want=("dx", "dgamma_pre", "dbeta_pre"))
    dtable = sbp.backward_embedding(g0["dx"], tokens, V, idx=idx, scale=SCALE)
    return dict(x1=x1, z1=z1, table=dtable, g0=g0["dgamma_pre"], b0=g0["dbeta_pre"], Wqkv=dWqkv, Wo=dWo, gate=g["dgate"], gp=g["dgamma_post"],
                bp=g["dbeta_post"], gn=g["dgamma_pre"], bn=g["dbeta_pre"])


def _oracle(p, tokens, doc, slopes, dx1, dz1, idx):
    """The same in 64 bits: the definitions of the steps, one behind the other."""
    p = {k: v.double().numpy() for k, v in p.items()}
    tokens, doc, slopes, dx1, dz1 = tokens.numpy(), doc.numpy(), slopes.double().numpy(), dx1.double().numpy(), dz1.double().numpy()
    pos = np.arange(N)
    attn = dict(scale=float(np.float32(D ** -0.5)), cap=CAP, slopes=slopes, causal=True)

    def parts(t, rows, b):
        x = t[b * rows:(b + 1) * rows].reshape(rows, H + 2 * HK, D)
        return x[:, :H], x[:, H:H + HK], x[:, H + HK:]
    x0 = lm.embedding(tokens, p["table"], float(np.float32(SCALE)))
    _, z0 = lm.residual_norm(x0, None, KIND, EPS, gamma_pre=p["g0"], beta_pre=p["b0"])
    qkv = z0 @ p["Wqkv"].T
    outs = [lm.attention(*parts(qkv, N, b), pos, doc=doc[b * N:(b + 1) * N], **attn) for b in range(B)]
    A, lse = np.concatenate([o[0].reshape(N, -1) for o in outs]), np.concatenate([o[1] for o in outs])
    y = A @ p["Wo"].T
    step = dict(alpha=ALPHA, gate=p["gate"], gamma_post=p["gp"], beta_post=p["bp"], gamma_pre=p["gn"])
    x1, z1 = lm.residual_norm(x0, y, KIND, EPS, beta_pre=p["bn"], **step)
    g = lm.residual_norm_backward(dx1, dz1[idx], x1[idx], y[idx], idx, M, KIND, EPS, **step)
    dA = g["dy_k"] @ p["Wo"]
    nk, dqkv = len(idx) // B, []
    for b in range(B):
        at = idx[b * nk:(b + 1) * nk]
        q, k, v = parts(qkv[at], nk, 0)
        r = lm.attention_backward(q, k, v, A[at].reshape(nk, H, D), dA[b * nk:(b + 1) * nk].reshape(nk, H, D), lse[at], at - b * N, doc=doc[at], **attn)
        dqkv.append(np.concatenate([t.reshape(nk, -1) for t in r], axis=1))
    dqkv = np.concatenate(dqkv)
    g0 = lm.residual_norm_backward(g["dx"], dqkv @ p["Wqkv"], x0[idx], None, idx, M, KIND, EPS, gamma_pre=p["g0"])
    return dict(x1=x1, z1=z1, table=lm.embedding_backward(g0["dx"][idx], tokens[idx], V, float(np.float32(SCALE))), g0=g0["dgamma_pre"], b0=g0["dbeta_pre"],
                Wqkv=dqkv.T @ z0[idx], Wo=g["dy_k"].T @ A[idx], gate=g["dgate"], gp=g["dgamma_post"], bp=g["dbeta_post"], gn=g["dgamma_pre"],
                bn=g["dbeta_pre"])


def _autograd(p, tokens, doc, slopes, dx1, dz1):
    """The same model in 64 bits by automatic differentiation."""
    p = {k: v.double().requires_grad_() for k, v in p.items()}
    i = torch.arange(N)
    see = (doc.view(B, N, 1) == doc.view(B, 1, N)) & (i[None, :, None] >= i[None, None])
    x0 = SCALE * p["table"][tokens]

    def norm(x, g, b):
        x = x - x.mean(-1, keepdim=True)
        return x / (x.pow(2).mean(-1, keepdim=True) + EPS).sqrt() * g + b
    qkv = (norm(x0, p["g0"], p["b0"]) @ p["Wqkv"].T).view(B, N, H + 2 * HK, D).transpose(1, 2)
    q, k, v = qkv[:, :H], qkv[:, H:H + HK].repeat_interleave(H // HK, 1), qkv[:, H + HK:].repeat_interleave(H // HK, 1)
    s = CAP * torch.tanh(q @ k.transpose(2, 3) * D ** -0.5 / CAP) - slopes.double()[:, None, None] * (i[:, None] - i[None]).abs()
    A = torch.softmax(s.masked_fill(~see[:, None], -math.inf), -1) @ v
    y = A.transpose(1, 2).reshape(M, C) @ p["Wo"].T
    x1 = ALPHA * x0 + p["gate"].repeat_interleave(N, 0) * norm(y, p["gp"], p["bp"])
    z1 = norm(x1, p["gn"], p["bn"])
    torch.autograd.backward((x1, z1), (dx1.double(), dz1.double()))
    return dict({k: v.grad for k, v in p.items()}, x1=x1.detach(), z1=z1.detach())


def _held(got, ref):
    for k, r in ref.items():
        r, x = np.asarray(r), got[k].double().cpu().numpy()
        assert x.shape == r.shape and np.isfinite(x).all(), k
        assert np.abs(x - r).max() <= TOLERANCE * np.abs(r).max(), (k, float(np.abs(x - r).max()), float(np.abs(r).max()))


def _cuda(model):
    p, *rest = model
    return ({k: v.cuda() for k, v in p.items()}, *[t.cuda() for t in rest])


def test_every_token_kept_is_the_models_gradient():
    model = _model(1)
    got = _run(*_cuda(model), torch.arange(M, dtype=torch.int32, device="cuda"))
    _held(got, _autograd(*model))


@pytest.mark.parametrize("k", [1, 3])
def test_drawn_keep_sets(k):
    model = _model(2)
    idx, _ = sbp.sample_indices(B, 0, N, 1, k, seed=7, stream_id=k, mode=sbp.TEMPORAL, cell=4)
    assert idx.numel() == M * k // 4
    _held(_run(*_cuda(model), idx), _oracle(*model, idx.cpu().numpy()))


def test_bf16_runs_alike_twice_and_in_a_graph():
    """The bf16 path: the same bits on a second run and on every replay of a captured one, with eager runs in between."""
    p, tokens, doc, slopes, dx1, dz1 = _cuda(_model(3))
    p = {k: v.to(torch.bfloat16) if k in ("table", "Wqkv", "Wo") else v for k, v in p.items()}
    dx1, dz1 = dx1.to(torch.bfloat16), dz1.to(torch.bfloat16)
    idx, _ = sbp.sample_indices(B, 0, N, 1, 2, seed=9, stream_id=0, mode=sbp.TEMPORAL, cell=4)

    def run():
        return _run(p, tokens, doc, slopes, dx1, dz1, idx)
    first = {k: v.clone() for k, v in run().items()}
    assert all(torch.isfinite(v.float()).all() for v in first.values())
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = run()
    for _ in range(3):
        graph.replay()
        torch.cuda.synchronize()
        for k, v in first.items():
            assert torch.equal(v, held[k]), k
            held[k].zero_()
        again = run()
        assert all(torch.equal(v, again[k]) for k, v in first.items())
