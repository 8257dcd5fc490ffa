"""Host-side checks of the language-model entry points (include/sbp_lm.h): declared, exported, bound, and every bad argument refused
before anything touches a GPU (no call here launches a kernel)."""
import ctypes
import os
import re

import pytest
import torch

import paper_2210_00129_amd as sbp
from paper_2210_00129_amd import _lib

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = 4096                       # an address that is never read: validation comes first
OK, NULL, SHAPE, DTYPE, WORKSPACE, FLAGS = 0, -1, -2, -4, -6, -8


def test_every_declared_symbol_is_exported_and_bound():
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "sbp_lm.h")).read(), flags=re.S)
    names = sorted(set(re.findall(r"\b(sbp_[a-z_0-9]+)\s*\(", text)))
    assert names == sorted(_lib.LM_PROTOTYPES)
    handle = ctypes.CDLL(_lib.LIB_PATH)
    for n in names:
        assert hasattr(handle, n), n


def _attn(**kw):
    base = dict(B=2, n=10, h=4, h_kv=2, d=64, causal=1, scale=0.125, cap=0.0, slopes=None, doc=None, prefix=None)
    base.update(kw)
    return _lib.AttentionDesc(*base.values())


BAD_ATTENTION = [(dict(B=0), SHAPE), (dict(n=0), SHAPE), (dict(h=0), SHAPE), (dict(h_kv=0), SHAPE), (dict(h_kv=3), SHAPE), (dict(d=48), SHAPE),
                 (dict(d=256), SHAPE), (dict(causal=2), FLAGS), (dict(scale=float("nan")), SHAPE), (dict(scale=float("inf")), SHAPE),
                 (dict(cap=-1.0), SHAPE), (dict(cap=float("inf")), SHAPE), (dict(causal=0, prefix=P), FLAGS), (dict(B=1 << 16, n=1 << 16), SHAPE),
                 (dict(B=1 << 12, n=1 << 14, h=128, h_kv=128, d=16), SHAPE)]


@pytest.mark.parametrize("kw,status", BAD_ATTENTION)
def test_attention_refuses_bad_descriptors(kw, status):
    L, d = _lib.lib(), _attn(**kw)
    assert L.sbp_forward_attention_masked(d, P, 1, P, P, None) == status
    assert L.sbp_backward_attention_masked_workspace(d, 1, 1) == 0
    assert L.sbp_backward_attention_masked(d, P, P, P, P, P, 1, 1, 2 * P, 4 * P, 1 << 40, None) == status
    assert L.sbp_last_error() != b""


def test_attention_refuses_bad_arguments():
    L, d = _lib.lib(), _attn()
    fwd = L.sbp_forward_attention_masked
    assert fwd(None, P, 1, P, P, None) == NULL
    assert fwd(d, P, 2, P, P, None) == DTYPE
    assert fwd(d, None, 1, P, P, None) == NULL and fwd(d, P, 1, None, P, None) == NULL
    assert fwd(d, P + 8, 1, P, P, None) == SHAPE and fwd(d, P, 1, P + 2, P, None) == SHAPE
    need = L.sbp_backward_attention_masked_workspace(d, 5, 1)
    bwd = L.sbp_backward_attention_masked
    good = [d, P, P, P, P, P, 5, 1, 2 * P, 4 * P, max(need, 1 << 30), None]

    def call(**kw):
        a = list(good)
        for k, v in kw.items():
            a[int(k[1:])] = v
        return bwd(*a)

    for i in (1, 2, 3, 4, 8):
        assert call(**{f"_{i}": None}) == NULL, i
    assert call(_5=None) == NULL                                  # idx, with n_k < n
    assert call(_6=11) == SHAPE and call(_6=-1) == SHAPE
    assert call(_7=3) == DTYPE
    assert call(_1=P + 4) == SHAPE and call(_8=P) == SHAPE        # alignment; the output is one of the inputs
    assert call(_6=0, _1=None) == OK                              # no kept token: nothing to do
    if need:
        assert call(_9=None) == WORKSPACE and call(_10=need - 1) == WORKSPACE and call(_9=4 * P + 128) == WORKSPACE


def _norm(**kw):
    base = dict(M=12, C=8, kind=0, G=1, alpha=1.0, eps=1e-5, reserved=0, gate=P, gamma_post=P, beta_post=P, gamma_pre=P, beta_pre=P)
    base.update(kw)
    return _lib.ResidualNormDesc(*base.values())


BAD_NORM = [(dict(M=0), SHAPE), (dict(M=1 << 31), SHAPE), (dict(C=0), SHAPE), (dict(C=16385), SHAPE), (dict(kind=2), FLAGS), (dict(G=0), SHAPE),
            (dict(G=5), SHAPE), (dict(M=70000, G=70000), SHAPE), (dict(alpha=float("nan")), SHAPE), (dict(eps=0.0), SHAPE), (dict(eps=float("inf")), SHAPE),
            (dict(reserved=1), FLAGS), (dict(gamma_post=None), NULL), (dict(gamma_pre=None), NULL)]


@pytest.mark.parametrize("kw,status", BAD_NORM)
def test_norms_refuse_bad_descriptors(kw, status):
    L, d = _lib.lib(), _norm(**kw)
    assert L.sbp_forward_residual_norm(d, P, P, 1, P, 2 * P, None) == status
    assert L.sbp_backward_residual_norm_workspace(d, 1, 1, 0) == 0
    assert L.sbp_backward_residual_norm(d, P, P, P, P, P, P, 1, 1, 2 * P, 3 * P, None, 4 * P, 1 << 40, 0, None) == status


def test_norms_refuse_bad_arguments():
    L, d = _lib.lib(), _norm()
    fwd = L.sbp_forward_residual_norm
    assert fwd(None, P, P, 1, P, P, None) == NULL and fwd(d, None, P, 1, P, 2 * P, None) == NULL and fwd(d, P, None, 1, P, 2 * P, None) == NULL
    assert fwd(d, P, P, 7, P, 2 * P, None) == DTYPE
    assert fwd(d, P, 2 * P, 1, None, P, None) == SHAPE and fwd(d, P, 2 * P, 1, 3 * P, 3 * P, None) == SHAPE     # z is x, z is x_out
    assert fwd(_norm(gamma_pre=None, beta_pre=None), P, 2 * P, 1, None, 3 * P, None) == NULL
    assert fwd(d, P, 2 * P, 1, None, None, None) == OK            # nothing wanted
    g = _lib.ResidualNormGrads(P, P, P, P, P)
    need = L.sbp_backward_residual_norm_workspace(d, 4, 1, 0)
    assert need > 0 and need % 256 == 0
    good = [d, P, 2 * P, 3 * P, 4 * P, P, P, 4, 1, 5 * P, 6 * P, g, 16 * P, need, 0, None]

    def call(**kw):
        a = list(good)
        for k, v in kw.items():
            a[int(k[1:])] = v
        return L.sbp_backward_residual_norm(*a)

    assert call(_3=None) == NULL and call(_4=None) == NULL and call(_5=None) == NULL and call(_2=None) == NULL
    assert call(_7=13) == SHAPE and call(_7=-1) == SHAPE
    assert call(_0=_norm(G=3)) == SHAPE                           # K is no multiple of G
    assert call(_8=5) == DTYPE and call(_14=1 | 2) == FLAGS
    assert call(_0=_norm(gate=None)) == NULL and call(_0=_norm(gamma_post=None, beta_post=None)) == NULL
    assert call(_0=_norm(gamma_pre=None, beta_pre=None)) == NULL
    assert call(_10=P) == SHAPE and call(_10=3 * P) == SHAPE and call(_9=2 * P) == SHAPE and call(_9=4 * P) == SHAPE and call(_10=5 * P) == SHAPE
    assert call(_12=None) == WORKSPACE and call(_13=need - 1) == WORKSPACE and call(_12=16 * P + 16) == WORKSPACE


def test_embedding_refuses_bad_arguments():
    L = _lib.lib()
    good = [P, 8, P, 6, 10, 8, 1.0, 1, 2 * P, None]

    def fwd(**kw):
        a = list(good)
        for k, v in kw.items():
            a[int(k[1:])] = v
        return L.sbp_forward_embedding(*a)

    assert fwd(_0=None) == NULL and fwd(_2=None) == NULL and fwd(_8=None) == NULL
    assert fwd(_1=2) == DTYPE and fwd(_7=4) == DTYPE
    assert fwd(_3=-1) == SHAPE and fwd(_4=0) == SHAPE and fwd(_4=1 << 30) == SHAPE and fwd(_5=0) == SHAPE and fwd(_6=float("inf")) == SHAPE
    assert fwd(_0=P + 4) == SHAPE and fwd(_3=0, _0=None) == OK
    need = L.sbp_backward_embedding_workspace(6, 4, 10, 8, 1, 0)
    base = [P, P, 8, P, 6, 4, 10, 8, 1.0, 1, 2 * P, 16 * P, max(need, 1 << 30), 0, None]

    def bwd(**kw):
        a = list(base)
        for k, v in kw.items():
            a[int(k[1:])] = v
        return L.sbp_backward_embedding(*a)

    assert bwd(_0=None) == NULL and bwd(_1=None) == NULL and bwd(_3=None) == NULL and bwd(_10=None) == NULL
    assert bwd(_2=1) == DTYPE and bwd(_9=2) == DTYPE
    assert bwd(_5=7) == SHAPE and bwd(_5=-1) == SHAPE and bwd(_4=1 << 31) == SHAPE and bwd(_8=float("nan")) == SHAPE
    assert bwd(_13=2) == FLAGS and bwd(_13=16) == FLAGS and bwd(_1=P + 2) == SHAPE
    for args in [(6, 7, 10, 8, 1, 0), (6, 4, 0, 8, 1, 0), (6, 4, 10, 8, 9, 0), (6, 4, 10, 8, 1, 2)]:
        assert L.sbp_backward_embedding_workspace(*args) == 0
    if need:
        assert bwd(_11=None) == WORKSPACE and bwd(_12=need - 1) == WORKSPACE


def test_binding_refuses_host_tensors():
    t = torch.zeros(4, 96)
    i = torch.zeros(4, dtype=torch.int32)
    for call in (lambda: sbp.forward_attention_masked(t, 2, 2, 16, 0.25), lambda: sbp.forward_residual_norm(t, t),
                 lambda: sbp.backward_attention_masked(t, t, t, t, 2, 2, 16, 0.25), lambda: sbp.forward_embedding(i, t),
                 lambda: sbp.backward_residual_norm(t, None, None, t, i, 4), lambda: sbp.backward_embedding(t, i, 10)):
        with pytest.raises(ValueError, match="GPU memory"):
            call()
    with pytest.raises(ValueError, match="one of"):
        sbp.backward_residual_norm(None, None, None, None, i, 4)


def test_attention_refuses_what_its_kernels_cannot_hold():
    L = _lib.lib()
    assert L.sbp_forward_attention_masked(_attn(cap=1025.0), P, 1, 2 * P, P, None) == SHAPE      # tanh to a few steps of fp32 of the cap
    assert L.sbp_backward_attention_masked_workspace(_attn(cap=1025.0), 5, 1) == 0
    assert L.sbp_backward_attention_masked_workspace(_attn(cap=1024.0), 5, 1) > 0
    assert L.sbp_forward_attention_masked(_attn(), P, 1, P, P, None) == SHAPE                    # the output is the input


def test_table_gradient_refuses_more_units_than_a_grid_has():
    L = _lib.lib()
    K, C = 1 << 25, 1 << 13
    assert L.sbp_backward_embedding_workspace(K, K, 1000, C, 1, 0) == 0
    assert L.sbp_backward_embedding(P, P, 4, None, K, K, 1000, C, 1.0, 1, P, 4 * P, 1 << 60, 0, None) == SHAPE
    assert L.sbp_backward_embedding_workspace(K, K - 32, 1000, C // 2, 1, 0) > 0
