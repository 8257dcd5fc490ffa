"""Helpers of the GPU tests of the language-model steps: the oracle per sample with element-wise error bounds.

The bounds follow the arithmetic.  u = 2^-24 is half a step of fp32; a rounding to bf16 is off by at most 2^-8 of the value.
Scores: z sums d products in fp32, so it is off by at most (d + 8) 2^-23 scale |q|.|k| (any order, fused or not); the score, its
bias, the cap's tanh, the difference to the row's maximum or lse and the exponential each add a few steps of fp32 of their size.
A weight P is thus off by delta = that sum, relatively, and in bf16 by another 2^-8 when it becomes an operand.  Sums over n terms
add at most 2 n 2^-24 of the sum of absolute terms.
"""
import math

import numpy as np
import torch

import paper_2210_00129_amd as sbp
from oracle import lm_oracle as lm

DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def out_step(dtype):
    return 2.0 ** -8 if dtype == "bf16" else 2.0 ** -24


def f64(t):
    return t.detach().cpu().double().numpy()


def within(got, ref, bound, what):
    """Every element of got is within bound of ref; infinities and zeros of the reference are met exactly where the bound is 0."""
    got, ref = f64(got) if torch.is_tensor(got) else got, np.asarray(ref)
    assert got.shape == ref.shape, (what, got.shape, ref.shape)
    fine = np.isfinite(ref)
    assert np.array_equal(fine, np.isfinite(got)) and np.array_equal(got[~fine], ref[~fine]), what
    over = np.abs(got - ref)[fine] - (1.01 * np.asarray(bound)[fine] + 1e-30)
    assert over.size == 0 or over.max() <= 0, (what, float(over.max()), float(np.abs(got - ref)[fine].max()))


class Case:
    """Random tensors of a masked attention, on the host, and the call's keyword arguments."""

    def __init__(self, B, n, h, hk, d, dtype, seed=0, cap=0.0, causal=False, slopes=False, doc=None, prefix=None, scale=None, spread=1.0):
        g = torch.Generator().manual_seed(seed)
        self.B, self.n, self.h, self.hk, self.d, self.dtype = B, n, h, hk, d, dtype
        self.qkv = (spread * torch.randn(B * n, (h + 2 * hk) * d, generator=g)).to(DT[dtype])
        self.dA = torch.randn(B * n, h * d, generator=g).to(DT[dtype])
        self.scale, self.cap, self.causal = 1.0 / math.sqrt(d) if scale is None else scale, cap, causal
        self.slopes = torch.tensor([0.3 / (i + 1) for i in range(h)]) if slopes else None
        self.doc = None if doc is None else torch.as_tensor(np.asarray(doc, dtype=np.int32).reshape(-1))
        self.prefix = None if prefix is None else torch.as_tensor(np.asarray(prefix, dtype=np.int32))

    def kw(self, device="cuda"):
        def dev(t):
            return None if t is None else t.to(device)
        return dict(B=self.B, h=self.h, d=self.d, scale=self.scale, h_kv=self.hk, cap=self.cap, causal=self.causal, slopes=dev(self.slopes),
                    doc=dev(self.doc), prefix=dev(self.prefix))

    def split(self, qkv, b, rows):
        """q, k, v of sample b in 64 bits; rows: tokens per sample in qkv."""
        x = f64(qkv[b * rows:(b + 1) * rows]).reshape(rows, self.h + 2 * self.hk, self.d)
        return x[:, :self.h], x[:, self.h:self.h + self.hk], x[:, self.h + self.hk:]

    def oracle_kw(self, b, pos):
        return dict(cap=float(np.float32(self.cap)), slopes=None if self.slopes is None else f64(self.slopes), causal=self.causal,
                    doc=None if self.doc is None else self.doc.numpy()[b * self.n + pos], prefix=0 if self.prefix is None else int(self.prefix[b]))

    def weights(self, b, q, k, pos, a, lse):
        """P, its relative error without the rounding to bf16, and the slope of the cap with its error, of head a."""
        kw = self.oracle_kw(b, pos)
        c = a // (self.h // self.hk)
        slope = 0.0 if kw["slopes"] is None else kw["slopes"][a]
        scale = float(np.float32(self.scale))
        s, T = lm.scores(q[:, a], k[:, c], pos, scale, kw["cap"], slope)
        see = lm.visible(pos, kw["doc"], self.causal, kw["prefix"])
        l = np.where(np.isfinite(lse[:, a]), lse[:, a], 0.0)[:, None]
        with np.errstate(over="ignore"):
            P = np.where(see, np.exp(np.where(see, s - l, 0.0)), 0.0)
        dz = (self.d + 8) * 2.0 ** -23 * abs(scale) * (np.abs(q[:, a]) @ np.abs(k[:, c]).T)
        dist = np.abs(pos[:, None] - pos[None])
        delta = dz + 2.0 ** -21 * (1.0 + np.abs(s) + slope * dist + np.abs(l) + kw["cap"])
        return P, delta, T, (2.0 ** -20 + 2 * dz / kw["cap"]) if kw["cap"] else 0.0


def check_forward(case, out=None):
    """Runs the forward and holds it to the oracle; returns (A, lse) on the GPU."""
    A, lse = sbp.forward_attention_masked(case.qkv.cuda(), **case.kw()) if out is None else out
    n, d, step, bf = case.n, case.d, out_step(case.dtype), 2.0 ** -8 if case.dtype == "bf16" else 0.0
    pos = np.arange(n)
    gotA, gotl = f64(A).reshape(case.B, n, case.h, d), f64(lse).reshape(case.B, n, case.h)
    for b in range(case.B):
        q, k, v = case.split(case.qkv, b, n)
        scale = float(np.float32(case.scale))
        rA, rl = lm.attention(q, k, v, pos, scale, **case.oracle_kw(b, pos))
        for a in range(case.h):
            P, delta, _, _ = case.weights(b, q, k, pos, a, rl)
            c = a // (case.h // case.hk)
            terms = 2 * n * 2.0 ** -24
            rel = (P * delta).sum(axis=1) + terms
            bound = (P * (bf + delta + terms)) @ np.abs(v[:, c]) + np.abs(rA[:, a]) * (rel[:, None] + step)
            within(gotA[b, :, a], rA[:, a], bound, ("A", b, a))
            within(gotl[b, :, a], rl[:, a], rel + 2.0 ** -22 * (1 + np.abs(np.where(np.isfinite(rl[:, a]), rl[:, a], 0.0))), ("lse", b, a))
    return A, lse


def check_backward(case, keep=None, run=None):
    """Runs the backward on the kept positions keep [B, n_k] (None: all) after the oracle's forward; returns dqkv on the GPU.
    run(qkv_k, A_k, dA_k, lse_k, idx): another call in the place of the plain one."""
    B, n, h, hk, d = case.B, case.n, case.h, case.hk, case.d
    all_kept = keep is None
    keep = np.tile(np.arange(n), (B, 1)) if all_kept else np.asarray(keep)
    nk = keep.shape[1]
    rows = (np.arange(B)[:, None] * n + keep).reshape(-1)
    scale = float(np.float32(case.scale))
    A, lse = np.zeros((B * n, h * d)), np.zeros((B * n, h))
    for b in range(B):
        pos = np.arange(n)
        oA, ol = lm.attention(*case.split(case.qkv, b, n), pos, scale, **case.oracle_kw(b, pos))
        A[b * n:(b + 1) * n], lse[b * n:(b + 1) * n] = oA.reshape(n, -1), ol
    at = torch.from_numpy(rows).long()
    qkv_k, dA_k = case.qkv[at].contiguous(), case.dA[at].contiguous()
    A_k, lse_k = torch.from_numpy(A)[at].to(DT[case.dtype]), torch.from_numpy(lse)[at].float()
    idx = None if all_kept else torch.from_numpy(rows.astype(np.int32)).cuda()
    ins = (qkv_k.cuda(), A_k.cuda(), dA_k.cuda(), lse_k.cuda())
    out = sbp.backward_attention_masked(*ins, n=n, idx=idx, **case.kw()) if run is None else run(*ins, idx)
    got = f64(out).reshape(B, nk, h + 2 * hk, d)
    step, bf = out_step(case.dtype), 2.0 ** -8 if case.dtype == "bf16" else 0.0
    for b in range(B):
        pos = keep[b]
        q, k, v = case.split(qkv_k, b, nk)
        g, o, l = (f64(t[b * nk:(b + 1) * nk]) for t in (dA_k, A_k, lse_k))
        g, o = g.reshape(nk, h, d), o.reshape(nk, h, d)
        ref = lm.attention_backward(q, k, v, o, g, l, pos, scale, **case.oracle_kw(b, pos))
        bounds = [np.zeros_like(t) for t in ref]
        for a in range(h):
            c = a // (h // hk)
            P, delta, T, eT = case.weights(b, q, k, pos, a, l)
            diff = g[:, a] @ v[:, c].T - (g[:, a] * o[:, a]).sum(axis=1, keepdims=True)
            e = (d + 8) * 2.0 ** -23 * (np.abs(g[:, a]) @ np.abs(v[:, c]).T + (np.abs(g[:, a]) * np.abs(o[:, a])).sum(axis=1, keepdims=True))
            dM = np.abs(P * diff * T * scale)
            terms = 2 * nk * 2.0 ** -24 * (h // hk)
            err = abs(scale) * (P * delta * np.abs(diff) * T + P * e * T + P * np.abs(diff) * eT) + (bf + terms) * dM
            bounds[0][:, a] += err @ np.abs(k[:, c])
            bounds[1][:, c] += err.T @ np.abs(q[:, a])
            bounds[2][:, c] += (P * (bf + delta + terms)).T @ np.abs(g[:, a])
        at0 = 0
        for name, r, bd in zip(("dq", "dk", "dv"), ref, bounds):
            within(got[b, :, at0:at0 + r.shape[1]], r, bd + step * np.abs(r), (name, b))
            at0 += r.shape[1]
    return out
