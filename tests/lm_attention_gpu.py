"""The masked attention's definition in 64 bits on the GPU, one head at a time, with the bounds of lm_util: for samples too long for the
oracle's loops."""
import torch

import paper_2210_00129_amd as sbp
from lm_util import DT


class Long:
    """One sample of n tokens with all that the calls take; kept: positions of the backward's tokens (None: all)."""

    def __init__(self, n, h, hk, d, dtype, seed=0, cap=0.0, causal=False, slopes=False, doc=None, prefix=None, scale=None, kept=None):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.n, self.h, self.hk, self.d, self.dtype, self.cap, self.causal = n, h, hk, d, dtype, float(torch.tensor(cap)), causal
        self.qkv = torch.randn(n, (h + 2 * hk) * d, generator=g, device="cuda").to(DT[dtype])
        self.dA = torch.randn(n, h * d, generator=g, device="cuda").to(DT[dtype])
        self.scale = float(torch.tensor(d ** -0.5 if scale is None else scale))
        self.slopes = torch.tensor([0.3 / (i + 1) for i in range(h)], device="cuda") if slopes else None
        self.doc = None if doc is None else torch.as_tensor(doc, dtype=torch.int32, device="cuda")
        self.prefix = None if prefix is None else torch.tensor([prefix], dtype=torch.int32, device="cuda")
        self.kept = torch.arange(n, device="cuda") if kept is None else torch.as_tensor(kept, device="cuda").long()
        self.idx = None if kept is None else self.kept.int()
        self.kw = dict(B=1, h=h, d=d, scale=self.scale, h_kv=hk, cap=self.cap, causal=causal, slopes=self.slopes, doc=self.doc, prefix=self.prefix)

    def head(self, x, a):
        return x.view(x.shape[0], -1, self.d)[:, a].double().contiguous()

    def pairs(self, q, k, a, pos):
        """(scores, visible, 1 - tanh^2, the scores' error) of the tokens at pos."""
        z = self.scale * (q @ k.t().contiguous())
        dz = (self.d + 8) * 2.0 ** -23 * abs(self.scale) * (q.abs() @ k.t().abs().contiguous())
        s, T = z, torch.ones_like(z)
        if self.cap:
            t = torch.tanh(z / self.cap)
            s, T = self.cap * t, 1 - t * t
        later = pos[None] - pos[:, None]
        far = torch.zeros_like(z)
        if self.slopes is not None:
            far = float(self.slopes[a]) * later.abs().double()
            s = s - far
        see = torch.ones_like(later, dtype=torch.bool)
        if self.causal:
            see = later <= 0
            if self.prefix is not None:
                see |= (pos < int(self.prefix))[None]
        if self.doc is not None:
            o = self.doc[pos]
            see &= (o[:, None] == o[None]) & (o >= 0)[:, None]
        return s, see, T, dz + 2.0 ** -21 * (1 + s.abs() + far + self.cap)

    def _bf(self):
        return 2.0 ** -8 if self.dtype == "bf16" else 0.0

    def _held(self, got, ref, bound, what):
        over = (got.double() - ref).abs() - (1.01 * (bound + max(self._bf(), 2.0 ** -24) * ref.abs()) + 1e-30)
        assert torch.isfinite(got).all() and float(over.max()) <= 0, (what, float(over.max()))

    def check_forward(self):
        A, lse = sbp.forward_attention_masked(self.qkv, **self.kw)
        self.hold_forward(A, lse)
        return A, lse

    def hold_forward(self, A, lse):
        pos, terms = torch.arange(self.n, device="cuda"), 2 * self.n * 2.0 ** -24
        for a in range(self.h):
            c = a * self.hk // self.h
            q, k, v = (self.head(self.qkv, i) for i in (a, self.h + c, self.h + self.hk + c))
            s, see, _, delta = self.pairs(q, k, a, pos)
            s = torch.where(see, s, -torch.inf)
            l = torch.logsumexp(s, 1)
            empty = ~see.any(1)
            P = torch.where(see, torch.exp(s - l[:, None]), 0.0)
            delta = P * (delta + 2.0 ** -21 * torch.where(empty, 0.0, l.abs())[:, None])
            rel, ref = delta.sum(1) + terms, P @ v
            self._held(self.head(A, a), ref, (P * (self._bf() + terms) + delta) @ v.abs() + ref.abs() * rel[:, None], ("A", a))
            got = lse[:, a].double()
            assert torch.equal(got == -torch.inf, empty)
            assert ((got - l)[~empty].abs() <= 1.01 * (rel + 2.0 ** -22 * (1 + l.abs()))[~empty]).all(), ("lse", a)

    def check_backward(self, A=None, lse=None):
        """On the kept tokens; A and lse (of all tokens): the forward's unless given."""
        if A is None:
            A, lse = sbp.forward_attention_masked(self.qkv, **self.kw)
        ins = [t[self.kept].contiguous() for t in (self.qkv, A, self.dA, lse)]
        out = sbp.backward_attention_masked(*ins, n=self.n, idx=self.idx, **self.kw)
        self.hold_backward(*ins, out)
        return out

    def hold_backward(self, qkv, A, dA, lse, out):
        """The kept tokens' gradients `out` to the definition on these inputs."""
        at, m, share = self.kept, len(self.kept), self.h // self.hk
        terms = 2 * m * 2.0 ** -24 * share
        for c in range(self.hk):
            k, v = self.head(qkv, self.h + c), self.head(qkv, self.h + self.hk + c)
            dk, dv, bk, bv = (torch.zeros_like(k) for _ in range(4))
            for a in range(c * share, (c + 1) * share):
                q, g, o = self.head(qkv, a), self.head(dA, a), self.head(A, a)
                l = lse[:, a].double()
                l = torch.where(l == -torch.inf, 0.0, l)[:, None]
                s, see, T, delta = self.pairs(q, k, a, at)
                P = torch.where(see, torch.exp(torch.where(see, s - l, 0.0)), 0.0)
                delta = delta + 2.0 ** -21 * l.abs()
                diff = g @ v.t().contiguous() - (g * o).sum(1, keepdim=True)
                e = (self.d + 8) * 2.0 ** -23 * (g.abs() @ v.t().abs().contiguous() + (g * o).abs().sum(1, keepdim=True))
                eT = 2.0 ** -20 + 2 * delta / self.cap if self.cap else 0.0
                dM = P * diff * T * self.scale
                err = abs(self.scale) * P * (delta * diff.abs() * T + e * T + diff.abs() * eT) + (self._bf() + terms) * dM.abs()
                ref = dM @ k
                self._held(self.head(out, a), ref, err @ k.abs(), ("dq", a))
                dk += dM.t().contiguous() @ q
                bk += err.t().contiguous() @ q.abs()
                dv += P.t().contiguous() @ g
                bv += (P * (self._bf() + delta + terms)).t().contiguous() @ g.abs()
            self._held(self.head(out, self.h + c), dk, bk, ("dk", c))
            self._held(self.head(out, self.h + self.hk + c), dv, bv, ("dv", c))
