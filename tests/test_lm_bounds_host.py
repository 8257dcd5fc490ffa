"""The bounds that the norms between blocks are held to, on the CPU: their values are the oracle's, results in fp32 meet them at every
number of channels, and a result that leaves out a mean or a projection does not."""
import numpy as np
import pytest
import torch

from lm_bounds import DT, EPS, NORM_LAYER, NORM_RMS, NormCase, f32
from oracle import lm_oracle as lm

CHANNELS = [7, 64, 96, 200, 512, 520, 768, 771, 1024, 1030, 2048, 2056, 4096, 5000, 8184, 8191, 8192, 8200, 12001, 16383, 16384]


def _np(t):
    return None if t is None else t.double().numpy()


def _oracle(c, idx):
    kw = {k: _np(v) for k, v in dict(c.vectors, gate=c.gate).items()}
    x, z = lm.residual_norm(_np(c.x), _np(c.y), c.kind, f32(EPS), alpha=c.alpha, **kw)
    kw.pop("beta_pre")
    back = lm.residual_norm_backward(_np(c.d_out), _np(c.dz)[idx] if c.pre else None, _np(c.x)[idx] if c.pre else None, _np(c.y)[idx], idx, c.M, c.kind, f32(EPS),
                                     alpha=c.alpha, **kw)
    back["dx"] = back["dx"][idx]
    return dict(x_out=x, z=z), back


@pytest.mark.parametrize("kind", [NORM_RMS, NORM_LAYER])
@pytest.mark.parametrize("post,pre,beta,G", [(True, True, True, 2), (True, True, False, 1), (False, True, True, 0), (True, False, True, 3)])
def test_values_are_the_oracles(kind, post, pre, beta, G):
    c = NormCase(12, 37, "f32", kind, post, pre, beta, G, device="cpu")
    idx = c.kept(4 // max(G, 1) + 1)
    fwd, back = _oracle(c, idx.numpy())
    for name, near in {**c.forward(), **c.backward(idx)}.items():
        want = fwd.get(name, back.get(name))
        assert np.allclose(near.v.numpy().reshape(np.shape(want)), want, rtol=1e-10, atol=1e-11), name


def _plain(c, idx):
    """The oracle's formulas in fp32, rounded to the case's type at the end."""
    def p(t):
        return None if t is None else t.float().numpy()
    kw = {k: p(v) for k, v in dict(c.vectors, gate=c.gate).items()}
    alpha, eps = np.float32(c.alpha), np.float32(EPS)
    x, z = lm.residual_norm(p(c.x), p(c.y), c.kind, eps, alpha=alpha, **kw)
    kw.pop("beta_pre")
    back = lm.residual_norm_backward(p(c.d_out), p(c.dz)[idx], p(c.x)[idx], p(c.y)[idx], idx, c.M, c.kind, eps, alpha=alpha, **kw)
    back["dx"] = back["dx"][idx]
    assert x.dtype == np.float32 and back["dx"].dtype == np.float32
    rows = {k: torch.from_numpy(v).to(DT[c.dtype]) for k, v in dict(x_out=x, z=z, dx=back["dx"], dy_k=back["dy_k"]).items()}
    return {**rows, **{k: torch.from_numpy(v) for k, v in back.items() if k.startswith(("dg", "db"))}}


@pytest.mark.parametrize("C", [1] + CHANNELS)
@pytest.mark.parametrize("kind", [NORM_RMS, NORM_LAYER])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_plain_arithmetic_in_32_bits_meets_them(C, kind, dtype):
    c = NormCase(6, C, dtype, kind, G=2, device="cpu")
    idx = c.kept(2)
    got = _plain(c, idx.numpy())
    for name, near in {**c.forward(), **c.backward(idx)}.items():
        assert c.excess(name, got[name], near) <= 0, name


@pytest.mark.parametrize("C", CHANNELS)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_missing_mean_or_projection_does_not(C, dtype):
    for kind in (NORM_RMS, NORM_LAYER):
        c = NormCase(6, C, dtype, kind, G=2, device="cpu")
        idx = c.kept(2)
        ref = c.backward(idx)
        for term, name in (("pre_projection", "dx"), ("post_projection", "dy_k"), ("pre_mean", "dx"), ("post_mean", "dy_k")):
            if kind == NORM_LAYER or "mean" not in term:
                wrong = c.backward(idx, keep={term: 0.0})[name].v
                assert c.excess(name, wrong.float().to(DT[dtype]), ref[name]) > 0, (kind, term)
    # a layer norm whose rows keep their mean, in the place of each norm
    ref, back = c.forward(), c.backward(idx)
    c.kind = NORM_RMS
    for name, near in c.forward().items():
        assert c.excess(name, near.v.float().to(DT[dtype]), ref[name]) > 0, name
    for name, near in c.backward(idx).items():
        if name != "dbeta_pre":
            assert c.excess(name, near.v.float().to(DT[dtype] if name in ("dx", "dy_k") else torch.float32), back[name]) > 0, name
