"""GPU parity of the embedding's gradient where a wavefront sums 16 and 32 sorted places, two and four groups of eight, as it does for training steps: sums that
go on from group to group, runs that begin in front of a tile and end in any of its groups.  Bars: those of test_gpu_embedding.py."""
import numpy as np
import pytest

from paper_2505_03803_amd import binding as B

import gpu_util as G
from test_gpu_embedding import SPREADS, check_gradient

torch = G.torch_()
# tokens, vocabulary, columns, sorted places of a wavefront: the number of tokens is not a multiple of it; widths that whole pieces fit and others
SIZES = [(4107, 300, 4096, 16), (4107, 40, 3585, 16), (8209, 900, 4096, 32), (8209, 30, 3587, 32), (16401, 2000, 2048, 32)]


@pytest.mark.parametrize("T,V,d,tile", SIZES)
def test_tiles_are_as_long(T, V, d, tile):
    """By the workspace: two or, of more than 8192 tokens, four lists, and two rows of sums for each tile."""
    lists = (4 if T > 8192 else 2) * ((4 * T + 15) // 16 * 16)
    assert B.rwkvq_embedding_backward_workspace_size(T, d) == lists + -(-T // tile) * 2 * d * 4
    assert T % tile


def runs(rng, T, V):
    """Runs of every length up to 70, one behind the other, so that they begin and end at every place of a tile."""
    lengths = rng.permutation(np.arange(1, 71).repeat(T // 2000 + 1))
    return rng.permutation(np.repeat(np.arange(len(lengths)) % V, lengths)[:T])


@pytest.mark.gpu
@pytest.mark.parametrize("T,V,d,tile", SIZES, ids=lambda v: str(v))
@pytest.mark.parametrize("spread", ["same", "few", "zipf", "padded", "runs"])
@pytest.mark.parametrize("added", [False, True])
def test_gradient(T, V, d, tile, spread, added):
    rng = np.random.default_rng(T + d)
    torch.manual_seed(T + d)
    dt = ["f16", "bf16", "f32"][(len(spread) + tile // 16 + added) % 3]
    tokens = runs(rng, T, V) if spread == "runs" else SPREADS[spread](rng, T, V)
    assert len(tokens) == T
    print(T, V, d, spread, added, dt, flush=True)
    check_gradient(tokens, T, V, d, dt, 0.3, added, d + (5 if d % 2 else 8))
