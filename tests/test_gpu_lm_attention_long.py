"""GPU parity of the masked attention on samples of several lists of tiles (more than 16384 tokens in the backward), whose fully visible
tiles make a stream of their own before the masked ones.  Scores have a deviation of 5, so that a query gives most of its weight to a few
keys anywhere among those it sees: a tile left out moves some results by their own size."""
import numpy as np
import pytest
import torch

from lm_attention_gpu import Long

pytestmark = pytest.mark.gpu
N = 17000


def _documents(n, lo, hi, seed):
    """Documents of lo .. hi tokens in a row, the last 200 tokens of none."""
    rng = np.random.default_rng(seed)
    ids = np.repeat(np.arange(n // lo + 1), rng.integers(lo, hi + 1, size=n // lo + 1))[:n].astype(np.int32)
    ids[n - 200:] = -1
    return ids


MODS = dict(causal=lambda: dict(causal=True), documents=lambda: dict(causal=True, doc=_documents(N, 300, 900, 1)),
            both_ways=lambda: dict(doc=_documents(N, 300, 900, 2), slopes=True), prefix=lambda: dict(causal=True, cap=20.0, prefix=9000),
            bias=lambda: dict(causal=True, cap=30.0, slopes=True))


@pytest.mark.parametrize("mods", MODS)
@pytest.mark.parametrize("d,h,hk", [(64, 4, 2), (128, 2, 1), (32, 2, 2)])
def test_several_lists(mods, d, h, hk):
    c = Long(N, h, hk, d, "bf16", seed=3, scale=5 * d ** -0.5, **MODS[mods]())
    c.check_backward(*c.check_forward())


@pytest.mark.parametrize("mods", MODS)
@pytest.mark.parametrize("d", [64, 128])
def test_several_lists_of_kept_tokens(mods, d):
    """16500 of 17000 tokens: the tiles' positions have gaps."""
    kept = np.sort(np.random.default_rng(5).choice(N, size=16500, replace=False))
    Long(N, 2, 1, d, "bf16", seed=4, scale=5 * d ** -0.5, kept=kept, **MODS[mods]()).check_backward()


@pytest.mark.parametrize("mods", ["documents", "prefix"])
def test_kept_tokens_of_several_lists_in_any_order(mods):
    """Tiles that hold tokens from everywhere: nothing is fully visible."""
    kept = np.random.default_rng(6).permutation(N)[:16500]
    Long(N, 2, 1, 64, "bf16", seed=5, scale=5 / 8, kept=kept, **MODS[mods]()).check_backward()
