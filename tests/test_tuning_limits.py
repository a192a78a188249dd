"""CPU-side checks of the ends of what the entry points accept: calls of more threads than one launch holds are refused before anything is
launched, whichever of their launches is the largest."""
import pytest

from paper_2505_03803_amd import binding as B

from test_tuning_abi import embedding_backward, forward, gradient, rows


# 2^17 tiles of 32 tokens, 128 times 512 columns each: joining their runs takes 256 threads for each, 2^32 in all
@pytest.mark.parametrize("kw", [dict(T=1 << 22, d=1 << 16, vocab=8), dict(T=1 << 22, d=(127 << 9) + 1, vocab=8), dict(T=1 << 21, d=1 << 17, vocab=8, acc=1)])
def test_embedding_gradients_of_too_many_threads(kw):
    assert embedding_backward(**kw) == B.ERR_SHAPE


# as many rows as an int holds: their number and a tile's rows together are more
@pytest.mark.parametrize("kw", [dict(n_tokens=2 ** 31 - 1), dict(n_tokens=2 ** 31 - 8), dict(n_tokens=2 ** 31 - 16, adapters=0x10000), dict(n_tokens=1 << 30)])
def test_adapters_of_too_many_rows(kw):
    few = dict(n=1, K=8, N=8)
    assert forward(rows(n_seqs=1, **kw), **few) == B.ERR_SHAPE
    assert gradient(rows(n_seqs=1, **kw), **few) == (B.ERR_SHAPE, 0)
