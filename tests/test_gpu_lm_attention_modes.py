"""GPU parity of the masked attention where the scores' arithmetic takes another of its kernels: scales of zero and below, caps above
those whose weights need no maximum."""
import numpy as np
import pytest
import torch

from lm_attention_gpu import Long
from lm_util import Case, check_backward, check_forward

pytestmark = pytest.mark.gpu


def _keep(n, nk, seed):
    return np.sort(np.random.default_rng(seed).choice(n, size=nk, replace=False))[None]


@pytest.mark.parametrize("scale", [0.0, -0.125, -1.5, 1e-30, -1e-30])
@pytest.mark.parametrize("mods", [dict(), dict(causal=True), dict(causal=True, cap=20.0), dict(causal=True, cap=90.0), dict(slopes=True), dict(cap=3.0, slopes=True)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_scales_of_zero_and_below(scale, mods, dtype):
    for n, d, h, hk in ((150, 64, 2, 1), (200, 128, 2, 2), (70, 16, 2, 1)):
        c = Case(1, n, h, hk, d, dtype, seed=31, scale=scale, **mods)
        check_forward(c)
        check_backward(c, _keep(n, n // 2, 31))


@pytest.mark.parametrize("d,n", [(128, 1200), (128, 100), (64, 900), (32, 500), (16, 300)])
@pytest.mark.parametrize("cap,scale", [(61.0, None), (100.0, 1.0), (500.0, 3.0)])
def test_caps_that_need_the_maximum(d, n, cap, scale):
    c = Long(n, 4, 2, d, "bf16", seed=32, causal=True, cap=cap, scale=scale)
    c.check_backward(*c.check_forward())


@pytest.mark.parametrize("d", [16, 64, 128])
@pytest.mark.parametrize("cap,size", [(60.0, 1e-13), (60.0, 1e-18), (45.0, 1e-18), (20.0, 1e-18)])
def test_small_values_of_rows_at_the_lower_cap(d, cap, size):
    """Every score of a row near -cap and values so small that exp(-cap) of them is below fp32's range."""
    c = Case(1, 300, 1, 1, d, "bf16", seed=33, causal=True, cap=cap)
    c.qkv[:, :d] = 40.0
    c.qkv[:, d:2 * d] = -40.0
    c.qkv[:, 2 * d:] *= size
    check_forward(c)


@pytest.mark.parametrize("d", [16, 32, 64, 128])
@pytest.mark.parametrize("mods", [dict(cap=20.0), dict(cap=60.0), dict(), dict(cap=80.0), dict(slopes=True)])
def test_a_token_that_sees_itself_alone_has_its_own_value(d, mods):
    """The rounding of the only weight must not reach the result: documents of one token (and a causal text's first)."""
    n = 200
    c = Case(2, n, 2, 1, d, "bf16", seed=34, causal=True, doc=np.stack([np.arange(n), np.arange(n) // 2]), **mods)
    A, _ = check_forward(c)
    v = c.qkv.view(2, n, 4, d)[:, :, 3]
    got = A.cpu().view(2, n, 2, d)
    for a in range(2):
        assert torch.equal(got[0, :, a], v[0]) and torch.equal(got[1, ::2, a], v[1, ::2])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("cap", [1e-44, 1e-39, 1e-30, 1e-6])
@pytest.mark.parametrize("scale", [None, 0.0, -1e6])
@pytest.mark.parametrize("n,d", [(20, 64), (150, 32), (150, 128)])
def test_smallest_caps(dtype, cap, scale, n, d):
    """scale / cap beyond fp32: a key whose product with the query is 0 has a score of 0."""
    c = Case(1, n, 2, 1, d, dtype, seed=35, causal=True, cap=cap, scale=scale)
    c.qkv[::3, :2 * d] = 0.0
    check_forward(c)
    check_backward(c)


@pytest.mark.parametrize("n", [1, 2, 7, 26, 32, 33])
@pytest.mark.parametrize("mods", [dict(), dict(slopes=True), dict(causal=True)])
@pytest.mark.parametrize("cap", [20.0, 50.0, 500.0])
def test_lse_of_few_keys_is_right_to_fp32(n, mods, cap):
    """bf16, capped: the scores' error, 2^-22 of the cap where tanh is taken from an exponential, does not average out over few keys.  Up to 32
    tokens lse is held to the steps of fp32 of its own size: z's products and sums, ten steps for tanh, bias and exponentials."""
    d = 64
    c = Long(n, 2, 2, d, "bf16", seed=36, cap=cap, **mods)
    _, lse = c.check_forward()
    pos = torch.arange(n, device="cuda")
    for a in range(2):
        q, k = c.head(c.qkv, a), c.head(c.qkv, 2 + a)
        s, see, _, _ = c.pairs(q, k, a, pos)
        z = (q.abs() @ k.abs().t().contiguous()) * c.scale
        far = 0.0 if c.slopes is None else float(c.slopes[a]) * (pos[None] - pos[:, None]).abs()
        step = 2.0 ** -24 * ((d + 8) * z + 10 * (s.abs() + far) + 10)
        want = torch.logsumexp(torch.where(see, s, -torch.inf), 1)
        bound = torch.where(see, step, 0.0).amax(1) + 2.0 ** -24 * (n + 8 + 4 * want.abs())
        assert n > 32 or ((lse[:, a].double() - want).abs() <= 1.01 * bound).all()
