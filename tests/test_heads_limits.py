"""CPU-side checks of the largest linear attention calls: those whose launches would hold 2^32 threads or more are refused by their shape, with
a workspace of 0; the next smaller ones are not.  (They are given an unaligned pointer, which is looked at after the shape: nothing is launched.)"""
import pytest

from paper_2505_03803_amd import binding as B
from test_heads_abi import FAKE, attention, attention_backward

# n_seqs, n_tokens, heads, channels, offsets, whether forward and backward fit
CALLS = [
    (1 << 18, 1 << 18, 64, 8, None, False, False), ((1 << 18) - 1, (1 << 18) - 1, 64, 8, None, True, False),      # single tokens: 256 threads each
    (1 << 19, 1 << 19, 16, 128, None, True, False),
    ((1 << 17) - 16, 1 << 17, 64, 8, FAKE, False, False), ((1 << 17) - 17, 1 << 17, 64, 8, FAKE, True, False),      # segments: 512, here 16 more than sequences
    (1 << 16, 1 << 17, 64, 128, None, False, False), ((1 << 16) - 1, (1 << 17) - 2, 64, 128, None, True, True),      # 512 for each half of 128 channels
    (87382, 87382, 64, 64, None, True, False), (87381, 87381, 64, 64, None, True, True),                              # backward: 768
    (1 << 18, 1 << 19, 16, 128, None, False, False), ((1 << 18) - 1, (1 << 19) - 2, 16, 72, None, True, True),
]


@pytest.mark.parametrize("n_seqs,n_tokens,H,D,offsets,forward,backward", CALLS)
def test_threads_of_a_launch(n_seqs, n_tokens, H, D, offsets, forward, backward):
    h = B.Heads(n_seqs, n_tokens, H, D, offsets=offsets)
    assert attention(h, out=FAKE + 2) == (B.ERR_ALIGN if forward else B.ERR_SHAPE)
    assert attention_backward(h, dr=FAKE + 2) == (B.ERR_ALIGN if backward else B.ERR_SHAPE)
    assert (B.rwkvq_linear_attention_backward_workspace_size(h) > 0) == backward
    if not forward:
        assert B.rwkvq_linear_attention_workspace_size(h) == 0
