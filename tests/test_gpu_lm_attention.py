"""GPU parity of the masked attention, forward and backward on the kept tokens, against the fp64 oracle."""
import numpy as np
import pytest
import torch

import paper_2210_00129_amd as sbp
from lm_util import DT, Case, check_backward, check_forward, f64

pytestmark = pytest.mark.gpu


def _docs(B, n, seed, pad=0, shuffled=False):
    rng = np.random.default_rng(seed)
    d = np.sort(rng.integers(0, max(2, n // 20), size=(B, n)), axis=1)
    if shuffled:
        d = rng.permutation(d.reshape(-1)).reshape(B, n)
    if pad:
        d[-1, n - pad:] = -1
    return d


def _keep(B, n, nk, seed, ordered=True):
    rng = np.random.default_rng(seed)
    k = np.stack([rng.choice(n, size=nk, replace=False) for _ in range(B)])
    return np.sort(k, axis=1) if ordered else k


SIZES = [  # B, n, h, hk, d, n_k
    (1, 1, 1, 1, 64, 1),
    (2, 2, 2, 1, 32, 1),
    (3, 31, 3, 3, 64, 17),
    (2, 33, 2, 2, 16, 32),
    (1, 64, 4, 2, 128, 33),
    (2, 65, 2, 1, 64, 64),
    (1, 129, 3, 1, 32, 65),
    (2, 197, 3, 3, 64, 99),
    (1, 200, 8, 2, 128, 129),
    (1, 300, 2, 2, 16, 257),
    (1, 385, 4, 1, 64, 200),
    (1, 700, 2, 1, 128, 390),
]


def _mods(i, B, n):
    """Masks and score changes that go round with the sizes, so that every size meets several and every one meets several sizes."""
    return [dict(), dict(causal=True), dict(causal=True, cap=30.0), dict(cap=2.0, slopes=True), dict(causal=True, slopes=True, doc=_docs(B, n, i)),
            dict(doc=_docs(B, n, i, pad=n // 3)), dict(causal=True, prefix=[n // (b + 2) for b in range(B)]),
            dict(causal=True, cap=5.0, slopes=True, doc=_docs(B, n, i, shuffled=True), prefix=[n // 2] * B)][i % 8]


CASES = [(s, i + j * 3, dt) for i, s in enumerate(SIZES) for j, dt in enumerate(("f32", "bf16", "bf16"))]


@pytest.mark.parametrize("size,mod,dtype", CASES)
def test_forward(size, mod, dtype):
    B, n, h, hk, d, _ = size
    check_forward(Case(B, n, h, hk, d, dtype, seed=mod, **_mods(mod, B, n)))


@pytest.mark.parametrize("size,mod,dtype", CASES)
def test_backward(size, mod, dtype):
    B, n, h, hk, d, nk = size
    check_backward(Case(B, n, h, hk, d, dtype, seed=mod, **_mods(mod, B, n)), _keep(B, n, nk, mod))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("mods", [dict(), dict(causal=True, slopes=True), dict(causal=True, cap=3.0, prefix=[40, 0])])
def test_all_tokens_kept_needs_no_index_list(dtype, mods):
    check_backward(Case(2, 130, 2, 1, 64, dtype, seed=5, **mods))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_kept_tokens_in_any_order(dtype):
    c = Case(2, 150, 4, 2, 64, dtype, seed=6, causal=True, slopes=True, doc=_docs(2, 150, 6, pad=20))
    check_backward(c, _keep(2, 150, 101, 6, ordered=False))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("prefix", [0, 1, 64, 100, 1000])
def test_prefix_lengths(dtype, prefix):
    c = Case(1, 100, 2, 2, 32, dtype, seed=7, causal=True, prefix=[prefix])
    check_forward(c)
    check_backward(c, _keep(1, 100, 50, 7))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rows_that_see_nothing_are_zero(dtype):
    n = 140
    doc = np.zeros((3, n), dtype=np.int32)
    doc[0, :] = -1                                       # a sample that is padding altogether
    doc[1, 70:] = -5
    c = Case(3, n, 2, 1, 64, dtype, seed=8, causal=True, cap=4.0, doc=doc)
    A, lse = check_forward(c)
    out = check_backward(c, _keep(3, n, 90, 8))
    pad = torch.from_numpy(doc.reshape(-1) < 0)
    as_int = torch.int16 if dtype == "bf16" else torch.int32
    assert (A.cpu()[pad].view(as_int) == 0).all() and (lse.cpu()[pad] == -np.inf).all()
    keep = (np.arange(3)[:, None] * n + _keep(3, n, 90, 8)).reshape(-1)
    assert (out.cpu()[pad[torch.from_numpy(keep)]].view(as_int) == 0).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,junk", [(100, float("nan")), (100, float("inf")), (333, float("nan"))])
def test_nothing_reaches_a_query_from_what_it_does_not_see(dtype, n, junk):
    """Padding rows, later tokens and other documents hold NaN or infinities: the rows that do not see them are as exact as with the
    ordinary numbers there."""
    doc = np.repeat([0, 1, 2, -1], [n // 4, n // 4, n // 4, n - 3 * (n // 4)])[None]
    c = Case(1, n, 2, 1, 64, dtype, seed=9, causal=True, slopes=True, doc=doc)
    bad = np.zeros(n, dtype=bool)
    bad[doc[0] == -1] = True
    bad[n // 4 + 5] = True                               # the sixth token of document 1: its later tokens see it
    hit = np.zeros(n, dtype=bool)
    hit[n // 4 + 5:2 * (n // 4)] = True
    kw = c.kw()
    rows = torch.from_numpy(bad)
    A0, l0 = sbp.forward_attention_masked(c.qkv.cuda(), **kw)
    dirty = c.qkv.clone()
    dirty[rows] = junk
    A1, l1 = sbp.forward_attention_masked(dirty.cuda(), **kw)
    assert torch.isnan(A1.cpu()[torch.from_numpy(hit)]).all()
    at = torch.from_numpy(hit).cuda()
    check_forward(c, out=(torch.where(at[:, None], A0, A1), torch.where(at[:, None], l0, l1)))
    # backward: a token's gradients are exact unless a dirty token sees it or it sees one
    touched = np.zeros(n, dtype=bool)
    touched[n // 4:2 * (n // 4)] = True

    def run(qkv, A, dA, lse, idx):
        dirty_qkv, dirty_dA = qkv.clone(), dA.clone()
        dirty_qkv[rows.cuda()] = junk
        dirty_dA[rows.cuda()] = junk
        want = sbp.backward_attention_masked(qkv, A, dA, lse, n=n, idx=idx, **kw)
        got = sbp.backward_attention_masked(dirty_qkv, A, dirty_dA, lse, n=n, idx=idx, **kw)
        return torch.where(torch.from_numpy(touched).cuda()[:, None], want, got)

    check_backward(c, run=run)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_large_scores(dtype):
    """Scores of some hundreds: the running maximum has to move, and single keys take all the weight."""
    c = Case(1, 260, 2, 2, 64, dtype, seed=10, causal=True, spread=12.0)
    check_forward(c)
    check_backward(c, _keep(1, 260, 130, 10))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_scores_at_the_cap(dtype):
    """Scores far beyond the cap, on both sides: weights between exp(-2 cap) and 1 of each other."""
    c = Case(1, 130, 2, 1, 32, dtype, seed=11, cap=50.0, spread=20.0)
    check_forward(c)
    check_backward(c, _keep(1, 130, 70, 11))


def test_rows_that_all_sit_at_the_lower_cap():
    """Every score of a row near -cap: the sum of the weights must not vanish."""
    n, d = 70, 32
    for cap in (50.0, 60.0, 80.0, 200.0):
        c = Case(1, n, 1, 1, d, "bf16", seed=12, cap=cap)
        c.qkv[:, :d] = 40.0
        c.qkv[:, d:2 * d] = -40.0
        check_forward(c)
        check_backward(c)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_same_bits_every_time_and_on_another_stream(dtype):
    c = Case(2, 300, 4, 2, 64, dtype, seed=13, causal=True, cap=20.0, slopes=True, doc=_docs(2, 300, 13))
    kw, qkv, dA = c.kw(), c.qkv.cuda(), c.dA.cuda()
    A, lse = sbp.forward_attention_masked(qkv, **kw)
    g = sbp.backward_attention_masked(qkv, A, dA, lse, **kw)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        A2, lse2 = sbp.forward_attention_masked(qkv, **kw)
        g2 = sbp.backward_attention_masked(qkv, A2, dA, lse2, **kw)
    s.synchronize()
    assert torch.equal(A, A2) and torch.equal(lse, lse2) and torch.equal(g, g2)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_captured_and_replayed(dtype):
    c = Case(2, 200, 2, 1, 64, dtype, seed=14, causal=True, slopes=True, doc=_docs(2, 200, 14, pad=30))
    kw, qkv, dA = c.kw(), c.qkv.cuda(), c.dA.cuda()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        A, lse = sbp.forward_attention_masked(qkv, **kw)
        g = sbp.backward_attention_masked(qkv, A, dA, lse, **kw)
    for seed in range(4):
        fresh = torch.randn(qkv.shape, generator=torch.Generator().manual_seed(seed)).to(DT[dtype])
        qkv.copy_(fresh.cuda())
        graph.replay()
        torch.cuda.synchronize()
        A2, lse2 = sbp.forward_attention_masked(qkv, **kw)
        g2 = sbp.backward_attention_masked(qkv, A2, dA, lse2, **kw)
        torch.cuda.synchronize()
        assert torch.equal(A, A2) and torch.equal(lse, lse2) and torch.equal(g, g2)


def test_two_calls_at_once_with_workspaces_of_their_own():
    c = [Case(2, 257, 4, 2, 64, "bf16", seed=15 + i, causal=True) for i in range(2)]
    alone = []
    for x in c:
        A, lse = sbp.forward_attention_masked(x.qkv.cuda(), **x.kw())
        alone.append((A, lse, sbp.backward_attention_masked(x.qkv.cuda(), A, x.dA.cuda(), lse, **x.kw())))
    ins = [(x.qkv.cuda(), x.dA.cuda()) for x in c]
    torch.cuda.synchronize()
    streams, outs = [torch.cuda.Stream() for _ in c], []
    for x, s, (q, g), (A, lse, _) in zip(c, streams, ins, alone):
        with torch.cuda.stream(s):
            outs.append(sbp.backward_attention_masked(q, A, g, lse, **x.kw()))
    torch.cuda.synchronize()
    for o, (_, _, w) in zip(outs, alone):
        assert torch.equal(o, w)


def test_offsets_beyond_32_bits():
    """2.4e9 elements of qkv: the last sample has the bits that it has alone."""
    B, n, h, d = 9000, 128, 12, 64
    g = torch.Generator(device="cuda").manual_seed(1)
    last = torch.randn(n, 3 * h * d, generator=g, device="cuda").bfloat16()
    qkv = torch.zeros(B * n, 3 * h * d, dtype=torch.bfloat16, device="cuda")
    qkv[-n:] = last
    A, lse = sbp.forward_attention_masked(qkv, B, h, d, 0.125, causal=True)
    A1, l1 = sbp.forward_attention_masked(last, 1, h, d, 0.125, causal=True)
    assert qkv.numel() > 2 ** 31 and torch.equal(A[-n:], A1) and torch.equal(lse[-n:], l1)
    dA = torch.zeros_like(A)
    dA[-n:] = torch.randn(n, h * d, generator=g, device="cuda").bfloat16()
    out = sbp.backward_attention_masked(qkv, A, dA, lse, B, h, d, 0.125, causal=True)
    assert torch.equal(out[-n:], sbp.backward_attention_masked(last, A1, dA[-n:].contiguous(), l1, 1, h, d, 0.125, causal=True))


def test_gradients_of_shared_heads_are_the_sums_of_their_own():
    """Query heads that share a key / value head: its gradient is the sum over calls with one query head each (fp32: to rounding)."""
    n, h, d = 150, 4, 32
    c = Case(1, n, h, 1, d, "f32", seed=20, causal=True)
    A, lse = sbp.forward_attention_masked(c.qkv.cuda(), **c.kw())
    out = f64(sbp.backward_attention_masked(c.qkv.cuda(), A, c.dA.cuda(), lse, **c.kw()))
    total = np.zeros((n, 2 * d))
    for a in range(h):
        cols = torch.cat([torch.arange(a * d, (a + 1) * d), torch.arange(h * d, (h + 2) * d)])
        one = sbp.backward_attention_masked(c.qkv[:, cols].contiguous().cuda(), A[:, a * d:(a + 1) * d].contiguous(),
                                            c.dA[:, a * d:(a + 1) * d].contiguous().cuda(), lse[:, a:a + 1].contiguous(), 1, 1, d, c.scale, causal=True)
        total += f64(one)[:, d:]
        assert np.abs(f64(one)[:, :d] - out[:, a * d:(a + 1) * d]).max() <= 1e-5 * np.abs(out).max()
    assert np.abs(out[:, h * d:] - total).max() <= 1e-5 * np.abs(total).max()


def test_the_binding_refuses_what_does_not_fit():
    q = torch.zeros(8, 96, device="cuda")
    for call, err in [(lambda: sbp.forward_attention_masked(q, 3, 2, 16, 0.25), ValueError),
                      (lambda: sbp.forward_attention_masked(q, 2, 2, 32, 0.25), ValueError),
                      (lambda: sbp.forward_attention_masked(q.half(), 2, 2, 16, 0.25), TypeError),
                      (lambda: sbp.forward_attention_masked(q, 2, 2, 16, 0.25, doc=torch.zeros(7, dtype=torch.int32, device="cuda")), ValueError),
                      (lambda: sbp.forward_attention_masked(q, 2, 2, 16, 0.25, doc=torch.zeros(8, dtype=torch.int64, device="cuda")), TypeError),
                      (lambda: sbp.forward_attention_masked(q, 2, 2, 16, 0.25, prefix=torch.zeros(2, dtype=torch.int32, device="cuda")), sbp.SbpError),
                      (lambda: sbp.forward_attention_masked(torch.zeros(8, 192, device="cuda")[:, ::2], 2, 2, 16, 0.25), ValueError)]:
        with pytest.raises(err):
            call()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", [32, 128])
def test_prefix_beyond_the_sample(dtype, d):
    c = Case(4, 197, 2, 1, d, dtype, seed=21, causal=True, prefix=[-2 ** 31, -1, 2 ** 31 - 1, 197])
    check_forward(c)
    check_backward(c, _keep(4, 197, 120, 21))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_largest_cap(dtype):
    c = Case(1, 150, 2, 1, 64, dtype, seed=22, causal=True, cap=1024.0, spread=3.0)
    check_forward(c)
    check_backward(c, _keep(1, 150, 90, 22))


@pytest.mark.parametrize("dtype,d,h,hk", [("bf16", 64, 2, 1), ("bf16", 128, 2, 2), ("bf16", 16, 3, 1), ("f32", 32, 1, 1)])
def test_one_long_sample_is_its_documents(dtype, d, h, hk):
    """17000 tokens in one sample (several lists of tiles) against the oracle on the 34 samples of 500 that its documents make."""
    B, n = 34, 500
    own = _docs(B, n, 23)
    c = Case(B, n, h, hk, d, dtype, seed=23, causal=True, slopes=True, doc=own)
    kw = dict(c.kw(), B=1, doc=(c.doc.view(B, n) + 1000 * torch.arange(B, dtype=torch.int32)[:, None]).reshape(-1).cuda())
    check_forward(c, out=sbp.forward_attention_masked(c.qkv.cuda(), **kw))
    check_backward(c, run=lambda q, A, g, l, idx: sbp.backward_attention_masked(q, A, g, l, **kw))
    check_backward(c, _keep(B, n, 333, 23), run=lambda q, A, g, l, idx: sbp.backward_attention_masked(q, A, g, l, n=B * n, idx=idx, **kw))


@pytest.mark.parametrize("d", [32, 128])
@pytest.mark.parametrize("mods", [dict(causal=True), dict(causal=True, cap=20.0, prefix=[9000]), dict(slopes=True)])
def test_long_samples_without_documents(d, mods):
    """9500 tokens: bf16 against the fp32 kernels, which share no tile code.  A weight is off by 2^-8 as an operand, an output by 2^-8 as it is
    stored, so A by at most 2^-7 of the weighted sum of |v| and 1 % of that for everything in fp32."""
    c = Case(1, 9500, 2, 1, d, "bf16", seed=24, **mods)
    kw, qkv = c.kw(), c.qkv.cuda()
    A, lse = sbp.forward_attention_masked(qkv, **kw)
    wide = qkv.float()
    fA, fl = sbp.forward_attention_masked(wide, **kw)
    wide[:, 3 * d:] = wide[:, 3 * d:].abs()
    size, _ = sbp.forward_attention_masked(wide, **kw)
    assert ((A.float() - fA).abs() <= 1.01 * 2.0 ** -7 * size).all()
    # lse: the scores' (d + 8) 2^-23 scale |q||k| of each side (|q||k| below 4 d here), and the sum's 9500 2^-24 with slack for exponentials
    assert ((lse - fl).abs() <= 2 * ((d + 8) * 4 * d * c.scale * 2.0 ** -23 + 9500 * 2.0 ** -22)).all()
