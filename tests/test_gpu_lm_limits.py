"""What the Python calls of the language-model steps refuse because a number does not fit the field that it goes into."""
import pytest
import torch

import paper_2210_00129_amd as sbp

pytestmark = pytest.mark.gpu


def test_channels_beyond_32_bits():
    """(a view of one element: nothing of this size is allocated)"""
    wide, tok = torch.zeros(1, 1, dtype=torch.bfloat16, device="cuda").expand(1, (1 << 32) + 8), torch.zeros(1, dtype=torch.int32, device="cuda")
    for call in (lambda: sbp.forward_embedding(tok, wide), lambda: sbp.backward_embedding(wide, tok, 5), lambda: sbp.forward_residual_norm(wide)):
        with pytest.raises(ValueError, match="too many channels"):
            call()


@pytest.mark.parametrize("flags", [1 << 32, 1 << 63, -1])
def test_flags_beyond_32_bits(flags):
    x, tok = torch.zeros(4, 8, device="cuda"), torch.zeros(4, dtype=torch.int32, device="cuda")
    with pytest.raises(ValueError, match="flags"):
        sbp.backward_embedding(x, tok, 5, flags=flags)
    with pytest.raises(ValueError, match="flags"):
        sbp.backward_residual_norm(x, None, None, x, tok, 4, flags=flags)


def test_gradients_that_leave_their_dict_during_the_call():
    """The dict of preallocated gradients gives up one of them while the next is looked up (a key of the same hash, whose comparison
    empties the entry): the call still owns what it took."""
    M, C = 6, 40
    x, idx = torch.randn(M, C, device="cuda"), torch.arange(M, dtype=torch.int32, device="cuda")
    gamma, gate = torch.ones(C, device="cuda"), torch.ones(C, device="cuda")
    args = dict(gate=gate, gamma_post=gamma, want=("dgate", "dgamma_post"))
    want = sbp.backward_residual_norm(x, None, None, x, idx, M, **args)

    class Taker(str):
        def __hash__(self):
            return hash("dgamma_post")

        def __eq__(self, other):
            grads.pop("dgate", None)
            return False
    grads = {Taker("taker"): None, "dgate": torch.empty(C, device="cuda")}
    got = sbp.backward_residual_norm(x, None, None, x, idx, M, grads=grads, **args)
    assert "dgate" not in grads
    assert torch.equal(got["dgate"], want["dgate"]) and torch.equal(got["dgamma_post"], want["dgamma_post"])
