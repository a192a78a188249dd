"""The masks that large tests compare with are the oracle's."""
import numpy as np
import pytest

from oracle import tuning_oracle as TO

import fast_masks


@pytest.mark.parametrize("seed,p,M,n,call", [((2 ** 60 + 7, 2 ** 33 - 2), 0.3, 9, 41, 3), ((-5, -1), 0.05, 3, 8, 0), ((1, 2 ** 64 - 1), 0.9, 2, 17, 5)])
def test_masks(seed, p, M, n, call):
    want, factor = TO.keep(seed, p, M, n, call)
    got, other = fast_masks.keep(seed, p, M, n, call)
    assert np.array_equal(got, want) and other == factor
