"""The oracle of dropout, embeddings and adapters against the generator's published vectors, explicit sums and differences."""
import numpy as np
import pytest

from oracle import tuning_oracle as TO


# the known answers that were published with the generator
@pytest.mark.parametrize("counter,key,want", [
    ((0, 0, 0, 0), (0, 0), (0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8)),
    ((0xFFFFFFFF,) * 4, (0xFFFFFFFF,) * 2, (0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD)),
    ((0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344), (0xA4093822, 0x299F31D0), (0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1)),
])
def test_generator(counter, key, want):
    assert tuple(TO.philox(counter, key)) == want


def test_share_of_what_stays():
    stays, factor = TO.keep((123, -1), 0.25, 50, 203)
    # 10150 draws: five standard deviations are 0.0215
    assert abs(stays.mean() - 0.75) < 0.0215 and factor == 1.0 / 0.75
    assert not np.array_equal(stays, TO.keep((123, -1), 0.25, 50, 203, call=1)[0])
    assert np.array_equal(TO.keep((123, 7), 0.25, 5, 20)[0], TO.keep((123, 6), 0.25, 5, 20, call=1)[0])
    assert TO.keep((1, 2), 0.0, 3, 9)[0].all() and not TO.keep((1, 2), 1.0, 3, 9)[0].any()


def test_embedding_gradient_is_the_transpose():
    rng = np.random.default_rng(0)
    tokens, table, dout = [3, 0, 3, -1, 7, 4], rng.standard_normal((6, 5)), rng.standard_normal((6, 5))
    out = TO.embedding(tokens, table, 2.0)
    assert not out[3].any() and not out[4].any() and np.array_equal(out[0], 2.0 * table[3])
    grad, _, count = TO.embedding_backward(tokens, dout, 6, 2.0)
    assert np.isclose((out * dout).sum(), (grad * table).sum()) and list(count) == [1, 0, 0, 2, 1, 0]


def test_adapter_gradients_are_differences():
    rng = np.random.default_rng(1)
    lens, ids, scales, seed, p = [3, 0, 4, 2, 1], [1, 0, -1, 1, 2], [0.5, 2.0, -1.0], (5, 9), 0.3
    M, K, N, r = 10, 11, 6, 3
    x, dy, a, b = rng.standard_normal((M, K)), rng.standard_normal((M, N)), rng.standard_normal((3, r, K)), rng.standard_normal((3, N, r))
    stays, factor = TO.keep(seed, p, M, K)

    def loss(x, a, b):
        return float((TO.adapters(TO.dropout(x, seed, p), a, b, lens, ids, scales)[0] * dy).sum())

    h = TO.adapters(TO.dropout(x, seed, p), a, b, lens, ids, scales)[1]
    dx, da, db = TO.adapters_backward(TO.dropout(x, seed, p), dy, h, a, b, lens, ids, scales, stays * factor)
    for at, grad in ((0, dx), (1, da), (2, db)):
        for _ in range(20):
            step = [np.zeros_like(v) for v in (x, a, b)]
            step[at] = rng.standard_normal(step[at].shape)
            moved = [(v + 1e-4 * d, v - 1e-4 * d) for v, d in zip((x, a, b), step)]
            # linear in x, a and b alone: a central difference is exact but for the rounding of two losses of some hundred terms
            slope = (loss(*(m[0] for m in moved)) - loss(*(m[1] for m in moved))) / 2e-4
            assert abs(slope - (grad * step[at]).sum()) < 1e-7
    assert not da[0].any() and not db[0].any() and not dx[3:7].any()
