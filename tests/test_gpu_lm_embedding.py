"""GPU parity of the token table's lookup and gradient.  Bounds: one product and one rounding for the lookup; a sum of k rows in fp32 and
one product for the gradient: (k + 2) 2^-24 of the sum of absolute terms, plus the rounding of a bf16 output."""
import numpy as np
import pytest
import torch

import paper_2210_00129_amd as sbp
from lm_util import DT, f64, out_step, within
from oracle import lm_oracle as lm

pytestmark = pytest.mark.gpu


def _tokens(kind, M, V, rng):
    if kind == "one":
        return np.full(M, V // 2)
    if kind == "zipf":
        return np.minimum(np.exp(rng.random(M) * np.log(V + 1.0)).astype(np.int64), V) - 1
    if kind == "outside":
        return rng.integers(-V, 2 * V, size=M)
    return rng.integers(0, V, size=M)


def _case(M, V, C, dtype, kind, seed=0, long_tokens=True):
    rng = np.random.default_rng(seed)
    tok = torch.from_numpy(_tokens(kind, M, V, rng))
    return (tok if long_tokens else tok.int()), torch.from_numpy(rng.standard_normal((V, C))).to(DT[dtype]), \
        torch.from_numpy(rng.standard_normal((M, C))).to(DT[dtype]), rng


CASES = [(1, 1, 8, "f32", "even"), (5, 3, 7, "bf16", "even"), (64, 10, 40, "bf16", "zipf"), (300, 1000, 200, "f32", "even"), (333, 50, 129, "bf16", "outside"),
         (1100, 3000, 64, "f32", "outside"), (1500, 7, 96, "bf16", "even"), (2500, 40000, 64, "bf16", "zipf"), (4097, 2047, 72, "f32", "zipf"),
         (5000, 2048, 40, "bf16", "one"), (9000, 100, 264, "bf16", "zipf"), (20000, 70000, 8, "f32", "even"), (70000, 3000, 16, "bf16", "zipf"),
         (3000, 4200, 2056, "bf16", "zipf"), (1030, 4097, 24, "f32", "one"), (40, 5000000, 8, "bf16", "even"), (2100, 5000000, 8, "f32", "even")]


@pytest.mark.parametrize("M,V,C,dtype,kind", CASES)
def test_lookup(M, V, C, dtype, kind):
    tok, table, _, _ = _case(M, min(V, 100000), C, dtype, kind, long_tokens=M % 2 == 0)
    E = sbp.forward_embedding(tok.cuda(), table.cuda(), 3.3)
    ref = lm.embedding(tok.numpy(), f64(table), float(np.float32(3.3)))
    within(E, ref, np.abs(ref) * (out_step(dtype) + 2.0 ** -24), "E")


def _check_gradient(got, tok, dE, V, scale, out_dtype, base=None):
    """Only the rows of tokens that occur are computed on the host; the others have to be +0 (or `base`)."""
    tok, got = tok.numpy(), got.cpu()
    ok = (tok >= 0) & (tok < V)
    rows, at = np.unique(tok[ok], return_inverse=True)
    d = f64(dE)[ok]
    ref, size = np.zeros((len(rows), d.shape[1])), np.zeros((len(rows), d.shape[1]))
    np.add.at(ref, at, d)
    np.add.at(size, at, np.abs(d))
    count = np.bincount(at, minlength=len(rows))[:, None] if len(rows) else np.zeros((0, 1))
    s = float(np.float32(scale))
    ref, bound = ref * s, abs(s) * size * (count + 2) * 2.0 ** -24
    if base is not None:
        ref = ref + f64(base)[rows]
        bound = bound + 2.0 ** -24 * np.abs(ref)
    within(got[rows], ref, bound + np.abs(ref) * out_step(out_dtype), "dtable")
    others = np.ones(V, dtype=bool)
    others[rows] = False
    others = torch.from_numpy(others)
    if base is None:
        assert (got[others].view(torch.int16 if out_dtype == "bf16" else torch.int32) == 0).all()
    else:
        assert torch.equal(got[others], base.cpu()[others])


@pytest.mark.parametrize("M,V,C,dtype,kind", CASES)
def test_gradient(M, V, C, dtype, kind):
    tok, _, _, rng = _case(M, 1, C, dtype, kind, long_tokens=M % 2 == 0)
    tok = torch.from_numpy(_tokens(kind, M, V, rng)).to(tok.dtype)
    dE = torch.from_numpy(rng.standard_normal((M, C))).to(DT[dtype])
    K = max(1, M * 2 // 3)
    idx = rng.permutation(M)[:K].astype(np.int32)                 # any order
    at = torch.from_numpy(idx).long()
    g = sbp.backward_embedding(dE.cuda(), tok.cuda(), V, idx=torch.from_numpy(idx).cuda(), scale=1.7)
    _check_gradient(g, tok[at], dE[at], V, 1.7, "f32")
    g2 = sbp.backward_embedding(dE[at].cuda(), tok.cuda(), V, idx=torch.from_numpy(idx).cuda(), scale=1.7, flags=sbp.FLAG_DY_COMPACT)
    assert torch.equal(g, g2)
    _check_gradient(sbp.backward_embedding(dE.cuda(), tok.cuda(), V), tok, dE, V, 1.0, "f32")
    if V <= 100000:
        h = sbp.backward_embedding(dE.cuda(), tok.cuda(), V, scale=0.5, flags=sbp.FLAG_DW_OUT_BF16)
        _check_gradient(h, tok, dE, V, 0.5, "bf16")
        for flags, out in ((sbp.FLAG_ACCUMULATE_DW, "f32"), (sbp.FLAG_ACCUMULATE_DW | sbp.FLAG_DW_OUT_BF16, "bf16")):
            base = torch.from_numpy(rng.standard_normal((V, C))).to(DT[out])
            a = sbp.backward_embedding(dE.cuda(), tok.cuda(), V, scale=2.0, flags=flags, dtable=base.cuda())
            _check_gradient(a, tok, dE, V, 2.0, out, base)


def test_no_kept_row():
    none = torch.empty(0, dtype=torch.int32, device="cuda")
    tok = torch.zeros(5, dtype=torch.int64, device="cuda")
    assert (sbp.backward_embedding(torch.empty(0, 16, device="cuda"), tok, 9, idx=none, flags=sbp.FLAG_DY_COMPACT) == 0).all()
    assert sbp.forward_embedding(tok[:0], torch.zeros(9, 16, device="cuda")).shape == (0, 16)


@pytest.mark.parametrize("M", [500, 6000])
def test_same_bits_every_time_and_captured(M):
    tok, table, dE, _ = _case(M, 3000, 264, "bf16", "zipf")
    tok, table, dE = tok.cuda(), table.cuda(), dE.cuda()

    def step():
        return sbp.forward_embedding(tok, table, 2.0), sbp.backward_embedding(dE, tok, 3000, scale=2.0)

    step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        E, g = step()
    for seed in range(4):
        tok.copy_(torch.from_numpy(_tokens("zipf", M, 3000, np.random.default_rng(seed))))
        graph.replay()
        torch.cuda.synchronize()
        E2, g2 = step()
        torch.cuda.synchronize()
        assert torch.equal(E, E2) and torch.equal(g, g2)


def test_odd_addresses_and_rows():
    """A gradient whose rows start off a 16-byte border."""
    tok, table, dE, _ = _case(200, 30, 40, "bf16", "even")
    room = torch.empty(200 * 40 + 1, dtype=torch.bfloat16, device="cuda")
    odd = room[1:].view(200, 40)
    odd.copy_(dE)
    assert torch.equal(sbp.backward_embedding(odd, tok.cuda(), 30), sbp.backward_embedding(dE.cuda(), tok.cuda(), 30))
    t = torch.empty(30 * 40 + 1, dtype=torch.bfloat16, device="cuda")[1:].view(30, 40)
    t.copy_(table)
    assert torch.equal(sbp.forward_embedding(tok.cuda(), t, 1.5), sbp.forward_embedding(tok.cuda(), table.cuda(), 1.5))


def test_offsets_beyond_32_bits():
    V, C = 300000, 8192
    table = torch.zeros(V, C, dtype=torch.bfloat16, device="cuda")
    table[-1] = 1.0
    E = sbp.forward_embedding(torch.tensor([V - 1, 0, V], device="cuda"), table, 2.0)
    assert (E[0] == 2).all() and (E[1:] == 0).all()
    del table
    g = sbp.backward_embedding(torch.ones(3, C, device="cuda"), torch.tensor([V - 1, 5, V - 1], device="cuda"), V)
    assert (g[-1] == 2).all() and (g[5] == 1).all() and float(g.sum()) == 3 * C


def test_the_binding_refuses_what_does_not_fit():
    tok, t = torch.zeros(4, dtype=torch.int64, device="cuda"), torch.zeros(6, 8, device="cuda")
    for call, err in [(lambda: sbp.forward_embedding(tok.float(), t), TypeError), (lambda: sbp.forward_embedding(tok.cpu(), t), ValueError),
                      (lambda: sbp.backward_embedding(t, tok, 6), ValueError),
                      (lambda: sbp.backward_embedding(t[:4], tok, 6, flags=sbp.FLAG_ACCUMULATE_DW), ValueError),
                      (lambda: sbp.backward_embedding(t[:4], tok, 6, dtable=t.bfloat16()), TypeError)]:
        with pytest.raises(err):
            call()


@pytest.mark.parametrize("M,V,C,dtype,kind", [(5000, 60000, 512, "bf16", "zipf"), (16000, 70000, 384, "f32", "outside")])
def test_gradient_of_a_table_that_takes_longer_to_clear_than_to_sort(M, V, C, dtype, kind):
    rng = np.random.default_rng(3)
    tok, dE = torch.from_numpy(_tokens(kind, M, V, rng)), torch.from_numpy(rng.standard_normal((M, C))).to(DT[dtype])
    got = sbp.backward_embedding(dE.cuda(), tok.cuda(), V, scale=1.7)
    _check_gradient(got, tok, dE, V, 1.7, "f32")


@pytest.mark.parametrize("M,V,C,dtype,kind", [(3, 67, 3493, "bf16", "even"), (120, 30, 1031, "bf16", "zipf"), (250, 7, 2050, "f32", "one"), (15, 15000, 346, "f32", "outside"),
                                              (200, 5000, 61, "bf16", "zipf")])
@pytest.mark.parametrize("shift", [0, 1])
def test_few_rows_of_many_channels(M, V, C, dtype, kind, shift):
    """Rows cut into slices of columns; outputs that start between two pieces of 16 bytes, whose neighbours stay as they are."""
    tok, table, dE, _ = _case(M, V, C, dtype, kind, seed=5)
    ref = lm.embedding(tok.numpy(), f64(table), float(np.float32(0.7)))
    E = torch.full((M * C + 16,), 7.0, dtype=DT[dtype], device="cuda")
    sbp.forward_embedding(tok.cuda(), table.cuda(), 0.7, out=E[shift:shift + M * C].view(M, C))
    within(E[shift:shift + M * C].view(M, C), ref, np.abs(ref) * (out_step(dtype) + 2.0 ** -24), "E")
    assert (E[:shift] == 7).all() and (E[shift + M * C:] == 7).all()
    for flags, out in ((0, "f32"), (sbp.FLAG_DW_OUT_BF16, "bf16")):
        got = torch.full((V * C + 16,), 7.0, dtype=DT[out], device="cuda")
        part = got[shift:shift + V * C].view(V, C)
        sbp.backward_embedding(dE.cuda(), tok.cuda(), V, scale=0.7, flags=flags, dtable=part)
        _check_gradient(part, tok, dE, V, 0.7, out)
        assert (got[:shift] == 7).all() and (got[shift + V * C:] == 7).all()
    base = torch.randn(V, C, device="cuda")
    got = torch.empty(V * C + 1, device="cuda")[shift:shift + V * C].view(V, C).copy_(base)
    sbp.backward_embedding(dE.cuda(), tok.cuda(), V, scale=0.7, flags=sbp.FLAG_ACCUMULATE_DW, dtable=got)
    _check_gradient(got, tok, dE, V, 0.7, "f32", base=base)
