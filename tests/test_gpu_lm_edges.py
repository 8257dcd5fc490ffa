"""Calls of the language-model steps at the edges of what they accept: document numbers and slopes of any size and sign, samples by the hundred
thousand, a million tokens in documents, no kept token, row numbers that come twice, gradients that nothing but the gate needs."""
import numpy as np
import pytest
import torch

import paper_2210_00129_amd as sbp
from lm_attention_gpu import Long
from lm_bounds import NORM_LAYER, NormCase
from lm_util import DT, Case, check_backward, check_forward

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", [32, 64, 128])
def test_documents_of_any_number(dtype, d):
    big, rng = 2 ** 31 - 1, np.random.default_rng(1)
    n = 260
    runs = [np.repeat([big, 0, big - 1, -1, big], [70, 30, 60, 40, 60]), rng.choice([0, big, big - 1, -1, -2 ** 31, 7], size=n),
            np.repeat([-1, big, -2 ** 31, 0], [64, 64, 68, 64]), np.full(n, big)]
    c = Case(4, n, 2, 1, d, dtype, seed=61, causal=True, slopes=True, doc=np.stack(runs))
    check_forward(c)
    check_backward(c, np.stack([np.sort(rng.choice(n, 150, replace=False)) for _ in range(4)]))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("mods", [dict(causal=True), dict(), dict(causal=True, cap=20.0), dict(causal=True, prefix=120)])
@pytest.mark.parametrize("d,n", [(64, 300), (128, 500), (16, 200)])
def test_slopes_of_any_sign(dtype, mods, d, n):
    """Scores that grow with the distance, or do not change with it; the bound takes the bias' size."""
    for slopes in ([-0.05, 0.0], [0.0, 0.5], [-0.4, 0.02]):
        c = Long(n, 2, 1, d, dtype, seed=62, **mods)
        c.slopes = torch.tensor(slopes, device="cuda")
        c.kw["slopes"] = c.slopes
        pairs = c.pairs

        def with_size(q, k, a, pos, pairs=pairs, c=c):
            s, see, T, delta = pairs(q, k, a, pos)
            return s, see, T, delta + 2.0 ** -20 * c.slopes[a].abs().double() * (pos[None] - pos[:, None]).abs()
        c.pairs = with_size
        c.check_backward(*c.check_forward())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,n,h", [(400000, 1, 1), (100000, 3, 2), (60000, 33, 1)])
def test_many_samples(dtype, B, n, h):
    d = 16
    g = torch.Generator(device="cuda").manual_seed(63)
    qkv, dA = torch.randn(B * n, 3 * h * d, generator=g, device="cuda").to(DT[dtype]), torch.randn(B * n, h * d, generator=g, device="cuda").to(DT[dtype])
    A, lse = sbp.forward_attention_masked(qkv, B, h, d, 0.25, causal=True)
    out = sbp.backward_attention_masked(qkv, A, dA, lse, B, h, d, 0.25, causal=True)
    for b in (0, B // 2 + 1, B - 1):                     # a sample alone has the bits that it has among the others
        at = slice(b * n, (b + 1) * n)
        A1, l1 = sbp.forward_attention_masked(qkv[at].contiguous(), 1, h, d, 0.25, causal=True)
        assert torch.equal(A[at], A1) and torch.equal(lse[at], l1)
        assert torch.equal(out[at], sbp.backward_attention_masked(qkv[at].contiguous(), A1, dA[at].contiguous(), l1, 1, h, d, 0.25, causal=True))
    if n == 1:
        v = qkv[:, 2 * h * d:]
        assert torch.equal(A, v) and (out[:, 2 * h * d:] == dA).all()


def test_a_million_tokens_in_documents():
    """One sample of 2^20 tokens in documents of 512 against 2048 samples of one document: the same sums in another order of tiles."""
    B, n, d, h = 2048, 512, 64, 2
    g = torch.Generator(device="cuda").manual_seed(64)
    qkv, dA = torch.randn(B * n, 3 * h * d, generator=g, device="cuda").bfloat16(), torch.randn(B * n, h * d, generator=g, device="cuda").bfloat16()
    doc = torch.arange(B, dtype=torch.int32, device="cuda").repeat_interleave(n)
    one, many = dict(B=1, h=h, d=d, scale=0.125, causal=True, doc=doc), dict(B=B, h=h, d=d, scale=0.125, causal=True)
    A, lse = sbp.forward_attention_masked(qkv, **one)
    A2, lse2 = sbp.forward_attention_masked(qkv, **many)
    assert torch.equal(lse == -torch.inf, lse2 == -torch.inf) and float((lse - lse2).abs().max()) <= 512 * 2.0 ** -22
    # (two roundings of the weights and two of the output: 2^-7 of the weighted sum of |v| each, at most the largest |v|)
    assert float((A.float() - A2.float()).abs().max()) <= 2.0 ** -6 * float(qkv[:, 2 * h * d:].abs().max())
    out, out2 = (sbp.backward_attention_masked(qkv, A2, dA, lse2, **kw) for kw in (one, many))
    scale = out2.float().abs().view(B, n, -1).amax(1, keepdim=True)
    assert float(((out.float() - out2.float()).abs().view(B, n, -1) / scale).max()) <= 2.0 ** -5


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_no_kept_token(dtype):
    h, d, n = 2, 32, 10
    e = lambda *s: torch.empty(*s, dtype=DT[dtype], device="cuda")
    out = sbp.backward_attention_masked(e(0, 3 * h * d), e(0, h * d), e(0, h * d), torch.empty(0, h, device="cuda"), 3, h, d, 0.2, n=n,
                                        idx=torch.empty(0, dtype=torch.int32, device="cuda"))
    assert out.shape == (0, 3 * h * d)


@pytest.mark.parametrize("K", [60, 3000, 30000])
@pytest.mark.parametrize("flags", ["", "accumulate"])
def test_table_gradient_of_rows_that_come_twice(K, flags):
    """Every row of idx counts as often as it stands there."""
    M, V, C = K, 500, 72
    g = torch.Generator(device="cuda").manual_seed(65)
    tok, dE = torch.randint(0, V, (M,), generator=g, device="cuda"), torch.randn(M, C, generator=g, device="cuda")
    idx = torch.randint(0, M, (K,), generator=g, device="cuda")
    base = torch.randn(V, C, generator=g, device="cuda")
    kw = dict(flags=sbp.FLAG_ACCUMULATE_DW, dtable=base.clone()) if flags else {}
    got = sbp.backward_embedding(dE, tok, V, idx=idx.int(), scale=-1.5, **kw)
    ref, size = (torch.zeros(V, C, dtype=torch.float64, device="cuda") for _ in range(2))
    ref.index_add_(0, tok[idx], -1.5 * dE.double()[idx])
    size.index_add_(0, tok[idx], 1.5 * dE.double()[idx].abs())
    ref, size = ref + (base.double() if flags else 0), size + (base.double().abs() if flags else 0)
    count = torch.bincount(tok[idx], minlength=V)[:, None]
    assert ((got - ref).abs() <= (count + 3) * 2.0 ** -24 * size + 1e-30).all()


@pytest.mark.parametrize("M,V,C,dtype", [(3000000, 50000, 24, "bf16"), (2500001, 90, 9, "f32"), (300, 60000000, 8, "f32"), (100, 60000000, 8, "bf16")])
def test_large_tables_and_many_rows(M, V, C, dtype):
    g = torch.Generator(device="cuda").manual_seed(66)
    tok, dE = torch.randint(0, V, (M,), generator=g, device="cuda"), torch.randn(M, C, generator=g, device="cuda").to(DT[dtype])
    got = sbp.backward_embedding(dE, tok, V, scale=0.5)
    count = torch.bincount(tok, minlength=V)
    seen = count.nonzero()[:, 0]
    at = torch.zeros(V, dtype=torch.long, device="cuda")
    at[seen] = torch.arange(len(seen), device="cuda")
    ref, size = (torch.zeros(len(seen), C, dtype=torch.float64, device="cuda") for _ in range(2))
    ref.index_add_(0, at[tok], 0.5 * dE.double())
    size.index_add_(0, at[tok], 0.5 * dE.double().abs())
    # (a token's rows in chunks of 32, the chunks in turn)
    adds = torch.minimum(count[seen], 34 + count[seen] // 32)[:, None]
    assert ((got[seen] - ref).abs() <= (adds + 3) * 2.0 ** -24 * size + 1e-30).all()
    got[seen] = 0
    assert not got.view(torch.int32).any()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("flags", [0, "compact"])
def test_gradients_that_need_no_block_output(dtype, flags):
    """Without a norm behind the block, dy needs the gate and t alone: y_k may be left out; and with nothing but dy and y wanted, dx too."""
    flags = sbp.FLAG_DX_COMPACT if flags else 0
    c = NormCase(40, 136, dtype, NORM_LAYER, post=False, pre=True, beta=False, G=2, alpha=-0.5)
    idx = c.kept(9)
    ref = c.backward(idx)
    kw, d = c.kw(False), c.d_out[idx] if flags else c.d_out
    for y in (None, c.y[idx]):
        got = sbp.backward_residual_norm(d, c.dz[idx], c.x[idx], y, idx.int(), c.M, flags=flags, want=("dy_k",), **kw)
        assert list(got) == ["dy_k"] and c.excess("dy_k", got["dy_k"], ref["dy_k"]) <= 0
    got = sbp.backward_residual_norm(d, c.dz[idx], c.x[idx], c.y[idx], idx.int(), c.M, flags=flags, want=("dgate", "dgamma_pre"), **kw)
    for name in ("dgate", "dgamma_pre"):
        assert c.excess(name, got[name], ref[name]) <= 0
    assert sbp.backward_residual_norm(d, c.dz[idx], c.x[idx], None, idx.int(), c.M, flags=flags, want=(), **kw) == {}
