"""Host-side checks of the sizes that the language-model entry points accept at most (no call here launches a kernel)."""
import pytest

from paper_2210_00129_amd import _lib

SHAPE = -2
MOST = (1 << 22) - 1           # B * h * ceil(n / 32) of one attention call


@pytest.mark.parametrize("B,h,n", [(MOST, 1, 1), (MOST, 1, 32), (1, 1, 1 << 24), (12, 349525, 31), (1398101, 3, 1), (7, 1, (1 << 24) - 31), (65535, 64, 1), (127, 1, 1 << 20)])
@pytest.mark.parametrize("dtype", [0, 1])
def test_attention_tables_are_reached_by_32_bits(B, h, n, dtype):
    """What the backward's kernel reads of its workspace by unsigned 32-bit offsets (statistics per head and token, positions and
    documents per token, samples padded to 64 tokens) ends below 2^32 bytes at the largest calls that are accepted."""
    assert 1 <= B * h * -(-n // 32) <= MOST
    d = _lib.AttentionDesc(B, n, h, h, 16, 1, 0.25, 0.0, None, None, None)
    need = _lib.lib().sbp_backward_attention_masked_workspace(d, n, dtype)
    tiles = B * -(-n // 64)
    tables = need - -(-tiles * 16 // 256) * 256          # (the ranges per tile lie behind them; h_kv = h: nothing else)
    assert 4 * (2 * h + 2) * tiles * 64 <= tables < 1 << 32


def test_attention_refuses_more():
    for B, h, n in ((1 << 22, 1, 1), (1 << 11, 1 << 11, 32), (1 << 10, 1 << 12, 1)):
        d = _lib.AttentionDesc(B, n, h, h, 16, 1, 0.25, 0.0, None, None, None)
        assert _lib.lib().sbp_backward_attention_masked_workspace(d, n, 1) == 0
        assert _lib.lib().sbp_forward_attention_masked(d, 4096, 1, 1 << 20, None, None) == SHAPE


def test_table_refuses_more_channels_than_its_kernels_count():
    """A lane's next column is an int: beyond 2^30 channels a step of 2048 would pass 2^31."""
    L = _lib.lib()
    for C in ((1 << 30) + 1, (1 << 31) - 1):
        assert L.sbp_forward_embedding(4096, 4, 1 << 40, 1, 1, C, 1.0, 1, 1 << 45, None) == SHAPE
        assert L.sbp_backward_embedding_workspace(300, 300, 1, C, 1, 0) == 0
        assert L.sbp_backward_embedding(1 << 40, 4096, 4, None, 1, 1, 1, C, 1.0, 1, 1 << 45, None, 0, 0, None) == SHAPE
    assert L.sbp_backward_embedding_workspace(300, 300, 1, 1 << 28, 1, 0) > 0
