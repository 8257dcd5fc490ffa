"""The steps between two blocks in 64 bits together with a bound of what their fp32 arithmetic may be off by.

Every number is a value and a bound of its error (first order and the products of errors), carried through the steps of the definition as
they are carried out: an operation adds U = 2^-24 of its result (half a step of fp32), and a sum over the channels of a row adds ADDS U of
the sum of its absolute terms.  ADDS counts the additions that one term goes through: at most 16 channels of a thread, 6 steps across a
wavefront, 16 wavefronts.  So the bounds do not grow with the number of channels.  Square root and division: a step each (2 U).
A sum over rows: the rows of one team in turn, its neighbours in the workgroup (3), one in 32 of the workgroups, 32 of these sums.
"""
import math

import numpy as np
import torch

U = 2.0 ** -24
ADDS = 16 + 6 + 16
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
STEP = {"f32": 0.0, "bf16": 2.0 ** -8}                      # the rounding of an output to its type
EPS = 1e-5
NORM_RMS, NORM_LAYER = 0, 1


class Near:
    """v: the exact value of what is computed; e: how far the computed one may be from it."""

    def __init__(self, v, e=None):
        self.v, self.e = v, torch.zeros_like(v) if e is None else e

    def _rounded(self, v, e):
        return Near(v, e + U * (v.abs() + e))

    def __add__(self, o):
        return self._rounded(self.v + o.v, self.e + o.e)

    def __sub__(self, o):
        return self._rounded(self.v - o.v, self.e + o.e)

    def __mul__(self, o):
        return self._rounded(self.v * o.v, self.v.abs() * o.e + o.v.abs() * self.e + self.e * o.e)

    def total(self, dim, adds):
        size = (self.v.abs() + self.e).sum(dim, keepdim=True)
        return Near(self.v.sum(dim, keepdim=True), self.e.sum(dim, keepdim=True) + adds * U * size)

    def mean(self, keep=1.0):
        """Over the channels of a row: the sum times 1 / C (rounded, and the product is).  keep 0: a mean left out."""
        inv = 1.0 / self.v.shape[1]
        t = self.total(1, ADDS)
        return Near(keep * t.v * inv, (t.e * (1 + 4 * U) + 2 * U * t.v.abs()) * inv)

    def inverse_root(self):
        """1 / sqrt(self)."""
        v = self.v.rsqrt()
        return Near(v, v * (0.5 * self.e / (self.v - self.e) * (1 + 1e-3) + 4 * U))

    def rows(self, at):
        return Near(self.v[at], self.e[at])


def f32(x):
    return float(np.float32(x))


def number(x, like):
    return Near(torch.full((1, 1), f32(x), dtype=torch.float64, device=like.device))


def statistics(x, kind):
    """(the row less its mean, 1 / deviation)."""
    if kind == NORM_LAYER:
        x = x - x.mean()
    return x, ((x * x).mean() + number(EPS, x.v)).inverse_root()


def norm(x, gamma, beta, kind):
    c, r = statistics(x, kind)
    out = c * r * gamma
    return out if beta is None else out + beta


class NormCase:
    """Tensors of the step between two blocks; rows with a mean, and gradients that are correlated with the normalised rows, so that the
    means and projections that the definitions take out are of the size of the rows."""

    def __init__(self, M, C, dtype, kind, post=True, pre=True, beta=True, G=1, alpha=0.7, seed=0, device="cuda"):
        g = torch.Generator(device=device).manual_seed(seed)
        self.M, self.C, self.dtype, self.kind, self.G, self.alpha, self.device = M, C, dtype, kind, G, f32(alpha), device
        self.post, self.pre, self.beta = post, pre, beta
        dt = DT[dtype]

        def randn(*s):
            return torch.randn(*s, generator=g, device=device)
        self.x, self.y, self.d_out = (0.8 + randn(M, C)).to(dt), (1.5 * randn(M, C) - 0.6).to(dt), randn(M, C).to(dt)
        hat = self.x.float() - (self.x.float().mean(1, keepdim=True) if kind == NORM_LAYER else 0.0)
        self.dz = (0.5 + randn(M, C) + 0.6 * hat).to(dt)
        self.vectors = dict(gamma_post=1 + 0.2 * randn(C) if post else None, beta_post=0.2 * randn(C) if post and beta else None,
                            gamma_pre=1 + 0.2 * randn(C) if pre else None, beta_pre=0.2 * randn(C) if pre and beta else None)
        self.gate = 0.6 + 0.2 * randn(G, C) if G else None

    def kept(self, per_group):
        """per_group rows of every group, ascending."""
        groups, rows = max(self.G, 1), self.M // max(self.G, 1)
        g = torch.Generator(device=self.device).manual_seed(self.M + per_group)
        pick = torch.rand(groups, rows, generator=g, device=self.device).argsort(1)[:, :per_group].sort(1).values
        return (pick + rows * torch.arange(groups, device=self.device)[:, None]).reshape(-1)

    def near(self, name, rows=None):
        t = self.vectors[name] if name in self.vectors else getattr(self, name)
        if t is None:
            return None
        t = t if rows is None else t[rows]
        return Near(t.double().reshape(1, -1) if t.dim() == 1 else t.double())

    def spread(self, rows):
        """The gate of `rows` rows, group by group."""
        return None if self.gate is None else Near(self.gate.double().repeat_interleave(rows // self.G, 0))

    # ---- the definitions ----
    def forward(self):
        u = self.near("y")
        if self.post:
            u = norm(u, self.near("gamma_post"), self.near("beta_post"), self.kind)
        if self.gate is not None:
            u = u * self.spread(self.M)
        x = self.near("x") * number(self.alpha, u.v) + u
        out = dict(x_out=x)
        if self.pre:
            out["z"] = norm(x, self.near("gamma_pre"), self.near("beta_pre"), self.kind)
        return out

    def backward(self, idx, keep=None):
        """keep: factors of the terms that take out a mean or a projection, by name (1; tests leave one out)."""
        keep = keep or {}
        K, per = len(idx), len(idx) // max(self.G, 1)
        t = self.near("d_out", idx)
        alpha = number(self.alpha, t.v)
        sums = {}
        if self.pre:
            dz, gn = self.near("dz", idx), self.near("gamma_pre")
            x, r = statistics(self.near("x", idx), self.kind)
            g, hat = dz * gn, x * r
            into = g - hat * ((g * x).mean(keep.get("pre_projection", 1.0)) * r)
            if self.kind == NORM_LAYER:
                into = into - g.mean(keep.get("pre_mean", 1.0))
            t = t + r * into
            sums["dgamma_pre"], sums["dbeta_pre"] = dz * hat, dz
        out = dict(dx=alpha * t)
        y = self.near("y", idx)
        hat = y
        if self.post:
            c, r = statistics(y, self.kind)
            hat = c * r
        gate, gp = self.spread(K), self.near("gamma_post")
        gg = gate if gp is None else gp if gate is None else gate * gp
        h = t if gg is None else t * gg
        if self.post:
            into = h - hat * (h * hat).mean(keep.get("post_projection", 1.0))
            if self.kind == NORM_LAYER:
                into = into - h.mean(keep.get("post_mean", 1.0))
            out["dy_k"] = r * into
        else:
            out["dy_k"] = h
        # parameters: sums over rows
        threads = 256 if self.C <= 512 else min(1024, 1 << max(7, math.ceil(math.log2(self.C / 8))))
        teams = 4 if self.C <= 512 else 1
        blocks = max(1, min(-(-per // teams), max(1, 262144 // threads // max(self.G, 1))))
        adds = -(-per // (blocks * teams)) + 3 + -(-blocks * max(self.G, 1) // 32) + 32 + 4
        if self.pre:
            out["dgamma_pre"] = sums["dgamma_pre"].total(0, adds)
            if self.beta:
                out["dbeta_pre"] = sums["dbeta_pre"].total(0, adds)
        s1, s2 = t * hat, t
        if self.gate is not None:
            def by_group(n):
                n = Near(n.v.view(self.G, per, self.C), n.e.view(self.G, per, self.C)).total(1, adds)
                return Near(n.v[:, 0], n.e[:, 0])
            d = by_group(s1) if gp is None else by_group(s1) * gp
            if self.post and self.beta:
                d = d + by_group(s2) * self.near("beta_post")
            out["dgate"] = d
            s1, s2 = s1 * gate, s2 * gate
        if self.post:
            out["dgamma_post"] = s1.total(0, adds)
            if self.beta:
                out["dbeta_post"] = s2.total(0, adds)
        return out

    def excess(self, name, got, ref):
        """How far an output is beyond its bound, at most (no more than 0: right).  Rows are rounded to the tensors' type."""
        got = got.double().reshape(ref.v.shape)
        step = STEP[self.dtype] if name in ("x_out", "z", "dx", "dy_k") else 0.0
        assert torch.isfinite(got).all(), name
        return float(((got - ref.v).abs() - (1.01 * (ref.e + step * (ref.v.abs() + ref.e)) + 1e-30)).max())

    # ---- the calls' arguments ----
    def kw(self, beta_pre):
        d = dict(self.vectors, gate=self.gate, kind=self.kind, eps=EPS, alpha=self.alpha)
        if not beta_pre:
            d.pop("beta_pre")
        return d

    def wanted(self):
        return ["dx", "dy_k"] + ["dgate"] * (self.gate is not None) + ["dgamma_post"] * self.post + ["dbeta_post"] * (self.post and self.beta) + \
            ["dgamma_pre"] * self.pre + ["dbeta_pre"] * (self.pre and self.beta)
