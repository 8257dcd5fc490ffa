"""The masked attention where tensors hold infinities and NaN: they reach the results that see them, and no others, in a time of the order of
an ordinary call's."""
import numpy as np
import pytest
import torch

import paper_2210_00129_amd as sbp
from lm_util import DT, Case, check_backward, check_forward
from oracle import lm_oracle as lm

pytestmark = pytest.mark.gpu
MODS = [dict(causal=True), dict(), dict(causal=True, cap=20.0), dict(causal=True, cap=80.0, slopes=True), dict(docs=True), dict(docs=True, causal=True, slopes=True)]


def _case(n, d, h, hk, dtype, mods, seed):
    mods = dict(mods)
    if mods.pop("docs", False):
        ids = np.repeat([0, 1, 2, -1], [n // 4, n // 3, n - n // 4 - n // 3 - n // 8, n // 8])
        mods["doc"] = ids[None]
    return Case(1, n, h, hk, d, dtype, seed=seed, **mods)


def _visible(c):
    pos = np.arange(c.n)
    return lm.visible(pos, None if c.doc is None else c.doc.numpy(), c.causal, 0)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,d,h,hk", [(70, 16, 2, 1), (333, 32, 2, 2), (333, 64, 4, 2), (700, 128, 2, 1), (90, 128, 2, 2)])
@pytest.mark.parametrize("mods", MODS)
def test_single_values_of_v(dtype, n, d, h, hk, mods):
    """Single channels of v: the outputs of these channels that see them are infinite or NaN, everything else is as exact as ever."""
    c = _case(n, d, h, hk, dtype, mods, 41)
    inf, nan = float("inf"), float("nan")
    spots = [(3, 0, 5, inf), (n // 2, 0, 5, -inf), (n // 3, hk - 1, d - 1, -inf), (n - 1, 0, 0, nan), (n - 2, hk - 1, 7, inf), (n // 2 + 9, 0, 2, inf), (n // 2 + 9, 0, 3, nan)]
    see, want = _visible(c), np.zeros((n, h, d))
    dirty = c.qkv.clone()
    with np.errstate(invalid="ignore"):
        for j, kv, ch, value in spots:
            dirty[j, (h + hk + kv) * d + ch] = value
            for a in range(kv * (h // hk), (kv + 1) * (h // hk)):
                want[see[:, j], a, ch] += value
    hit = ~np.isfinite(want)
    assert hit.any()
    A0, _ = sbp.forward_attention_masked(c.qkv.cuda(), **c.kw())
    A, lse = sbp.forward_attention_masked(dirty.cuda(), **c.kw())
    got = A.float().cpu().numpy().reshape(n, h, d)
    assert np.array_equal(got[hit], want[hit].astype(np.float32), equal_nan=True)
    check_forward(c, out=(torch.where(torch.from_numpy(hit.reshape(n, -1)).cuda(), A0, A), lse))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,d,h,hk", [(70, 16, 2, 1), (333, 32, 2, 2), (333, 64, 4, 2), (430, 128, 2, 1)])
@pytest.mark.parametrize("mods", MODS)
@pytest.mark.parametrize("junk", [float("nan"), float("inf")])
def test_whole_tokens(dtype, n, d, h, hk, mods, junk):
    """Tokens of NaN or infinities, padding among them: a token that sees none and is seen by none has its ordinary results, one that sees a
    NaN has none."""
    c = _case(n, d, h, hk, dtype, mods, 42)
    bad = np.zeros(n, dtype=bool)
    if c.doc is not None:
        bad |= c.doc.numpy() < 0
        bad[n // 4 + 6] = True
    else:
        bad[[n - 3, n - 40 if n > 300 else n - 5]] = True
    see, kw, rows = _visible(c), c.kw(), torch.from_numpy(bad)
    sees = (see & bad[None]).any(axis=1)
    touched = sees | (see & bad[:, None]).any(axis=0)
    assert touched.any() and (c.doc is None or not touched.all())
    A0, l0 = sbp.forward_attention_masked(c.qkv.cuda(), **kw)
    dirty = c.qkv.clone()
    dirty[rows] = junk
    A, lse = sbp.forward_attention_masked(dirty.cuda(), **kw)
    at = torch.from_numpy(sees).cuda()
    if junk != junk:
        assert torch.isnan(A[at]).all()
    check_forward(c, out=(torch.where(at[:, None], A0, A), torch.where(at[:, None], l0, lse)))

    def run(qkv, A, dA, lse, idx):
        dq, dg = qkv.clone(), dA.clone()
        dq[rows.cuda()] = junk
        dg[rows.cuda()] = junk
        want = sbp.backward_attention_masked(qkv, A, dA, lse, n=n, idx=idx, **kw)
        got = sbp.backward_attention_masked(dq, A, dg, lse, n=n, idx=idx, **kw)
        if junk != junk:
            assert torch.isnan(got[at][:, :h * d]).all()
        return torch.where(torch.from_numpy(touched).cuda()[:, None], want, got)
    check_backward(c, run=run)


@pytest.mark.parametrize("d,cap,size", [(64, 50.0, 1e20), (128, 55.0, 1e18), (16, 0.0, 2e38), (128, 0.0, 2e38), (32, 100.0, 2e38)])
def test_sums_that_would_overflow(d, cap, size):
    """Values of v so large that a weight above 1 takes their sum beyond fp32: the result is their weighted mean all the same."""
    c = Case(1, 150, 2, 1, d, "bf16", seed=43, causal=True, cap=cap, spread=2.0)
    v = c.qkv[:, 3 * d:].float()
    c.qkv[:, 3 * d:] = (v.sign() * size * (0.5 + 0.5 * v.abs().clamp(max=1.0))).to(DT["bf16"])
    check_forward(c)


def _time(f):
    f()
    a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    best = float("inf")
    for _ in range(3):
        a.record()
        f()
        b.record()
        b.synchronize()
        best = min(best, a.elapsed_time(b))
    return best


@pytest.mark.parametrize("where", ["a token that most see", "one value of v", "everything", "padding", "padding, both ways"])
@pytest.mark.parametrize("dtype,n,h,hk,d", [("bf16", 2048, 16, 2, 128), ("bf16", 2048, 12, 12, 64), ("f32", 1024, 8, 8, 64)])
def test_they_cost_a_few_ordinary_calls(where, dtype, n, h, hk, d):
    """(a row at a time it was 30 to 340 calls)"""
    g = torch.Generator(device="cuda").manual_seed(44)
    qkv = torch.randn(n, (h + 2 * hk) * d, generator=g, device="cuda").to(DT[dtype])
    dA = torch.randn(n, h * d, generator=g, device="cuda").to(DT[dtype])
    doc = torch.zeros(n, dtype=torch.int32, device="cuda")
    if "padding" in where:
        doc[-92:] = -1
    kw = dict(B=1, h=h, h_kv=hk, d=d, scale=d ** -0.5, causal="both" not in where, doc=doc)
    A, lse = sbp.forward_attention_masked(qkv, **kw)
    plain = _time(lambda: sbp.forward_attention_masked(qkv, **kw)), _time(lambda: sbp.backward_attention_masked(qkv, A, dA, lse, n=n, **kw))
    bad, gbad = qkv.clone(), dA.clone()
    rows = dict(everything=slice(0, None)).get(where, slice(-92, None) if "padding" in where else slice(5, 6))
    if where == "one value of v":
        bad[rows, (h + hk) * d + 3] = float("inf")
    else:
        bad[rows] = float("nan")
        gbad[rows] = float("nan")
    A2, lse2 = sbp.forward_attention_masked(bad, **kw)
    with_them = _time(lambda: sbp.forward_attention_masked(bad, **kw)), _time(lambda: sbp.backward_attention_masked(bad, A2, gbad, lse2, n=n, **kw))
    assert with_them[0] < 24 * plain[0] and with_them[1] < 24 * plain[1], (plain, with_them)
