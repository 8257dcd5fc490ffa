"""GPU parity of the step between two blocks, held to bounds that do not grow with the channels (lm_bounds),
at every number of channels."""
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
