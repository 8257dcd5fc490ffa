"""GPU parity of the step between two blocks, held to bounds that do not grow with the channels (lm_bounds): more rows than the launch has
teams, so that every team takes several, crosses groups of the gate and adds up its rows; every number of channels; odd addresses."""
import pytest
import torch

import paper_2210_00129_amd as sbp
from lm_bounds import DT, NORM_LAYER, NORM_RMS, NormCase

pytestmark = pytest.mark.gpu
KINDS = [NORM_RMS, NORM_LAYER]


def _shifted(t):
    """The same rows one element off their place in memory."""
    room = torch.empty(t.numel() + 1, dtype=t.dtype, device=t.device)[1:].view(t.shape)
    return room.copy_(t)


def _check_forward(c, x=None, y=None, **outs):
    x_out, z = sbp.forward_residual_norm(c.x if x is None else x, c.y if y is None else y, **c.kw(True), **outs)
    assert (z is None) == (not c.pre)
    for name, near in c.forward().items():
        assert c.excess(name, dict(x_out=x_out, z=z)[name], near) <= 0, name


def _check_backward(c, idx, flags=0, shift=False):
    compact = flags & sbp.FLAG_DX_COMPACT
    move = _shifted if shift else lambda t: t
    d = move(c.d_out[idx] if compact else c.d_out)
    dz, x, y = (move(t[idx]) for t in (c.dz, c.x, c.y))
    outs = dict(dx=_shifted(d), dy_k=_shifted(y)) if shift else {}
    got = sbp.backward_residual_norm(d, dz if c.pre else None, x if c.pre else None, y, idx.int(), c.M, flags=flags, want=c.wanted(), **outs, **c.kw(False))
    ref = c.backward(idx)
    assert sorted(ref) == sorted(c.wanted())
    for name, near in ref.items():
        t = got[name][idx] if name == "dx" and not compact else got[name]
        assert c.excess(name, t, near) <= 0, name
    if not compact:
        dropped = torch.ones(c.M, dtype=torch.bool, device="cuda")
        dropped[idx] = False
        assert torch.equal(got["dx"][dropped], (c.alpha * c.d_out[dropped].float()).to(DT[c.dtype]))


# rows, channels, gates: a team of the forward has 2048 (8192 up to 512 channels) others
FORWARD = [(20000, 96, 5), (9000, 520, 3), (5000, 1030, 1), (4500, 2056, 2), (4300, 4100, 0), (4200, 8192, 1), (4200, 8200, 2), (2300, 12001, 1), (2100, 16384, 3)]


@pytest.mark.parametrize("M,C,G", FORWARD)
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_forward_of_several_rows_per_team(M, C, G, kind, dtype):
    _check_forward(NormCase(M, C, dtype, kind, G=G, seed=C))


# rows, channels, gates, kept rows per group: a team has 1023 (4095 up to 512 channels) to 255 others, split over the groups
BACKWARD = [(20000, 96, 5, 1900), (9000, 520, 3, 2100), (5000, 1030, 1, 2600), (3200, 2056, 2, 750), (2600, 4096, 1, 1300), (1400, 5000, 0, 640),
            (1200, 8184, 3, 190), (1400, 8191, 1, 650), (1400, 12001, 2, 300), (1300, 16384, 1, 600)]


@pytest.mark.parametrize("M,C,G,per_group", BACKWARD)
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("beta", [True, False])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_backward_of_several_rows_per_team(M, C, G, per_group, kind, beta, dtype):
    c = NormCase(M // max(G, 1) * max(G, 1), C, dtype, kind, beta=beta, G=G, seed=C)
    _check_backward(c, c.kept(per_group))


@pytest.mark.parametrize("M,C,K", [(300000, 64, 5), (40000, 1030, 7), (20000, 4100, 3), (18000, 8192, 2), (17000, 8200, 1)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_long_runs_of_dropped_rows(M, C, K, dtype):
    """More than 64 dropped rows for every team that passes them through."""
    c = NormCase(M, C, dtype, NORM_LAYER, G=0, seed=C)
    _check_backward(c, c.kept(K))


CHANNELS = [1, 7, 64, 96, 200, 512, 513, 768, 771, 1024, 1030, 2048, 2056, 4096, 4104, 5000, 8184, 8191, 8192, 8200, 12001, 16383, 16384]


@pytest.mark.parametrize("C", CHANNELS)
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("post,pre,beta,G", [(True, True, True, 2), (True, True, False, 1), (False, True, True, 0), (True, False, False, 3)])
def test_every_number_of_channels(C, kind, dtype, post, pre, beta, G):
    c = NormCase(30, C, dtype, kind, post, pre, beta, G, seed=C)
    _check_forward(c)
    idx = c.kept(5)
    _check_backward(c, idx)
    _check_backward(c, idx, flags=sbp.FLAG_DX_COMPACT)


@pytest.mark.parametrize("C", [136, 640, 1032, 2056, 5000, 8184, 12000, 16384])
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rows_of_whole_vectors_at_odd_addresses(C, kind, dtype):
    c = NormCase(24, C, dtype, kind, G=2, seed=C)
    x = _shifted(c.x)
    _check_forward(c, x=x, y=_shifted(c.y), x_out=_shifted(c.x), z=_shifted(c.x))
    idx = c.kept(5)
    _check_backward(c, idx, shift=True)
    _check_backward(c, idx, flags=sbp.FLAG_DX_COMPACT, shift=True)
