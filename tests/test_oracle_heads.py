"""Pins of the oracle of the multi-head block's operators: closed forms, invariants, and every gradient against central
differences in binary64."""
import numpy as np
import pytest

from oracle import block_oracle as BO
from oracle import heads_oracle as HO


def test_norm_by_hand():
    y, mean, rstd = HO.layer_norm(np.array([[1.0, 3.0], [5.0, 5.0]]), np.array([2.0, 10.0]), np.array([0.5, 1.0]), eps=3.0)
    # row 0: mean 2, variance 1, rstd 1/2; row 1: no deviation
    assert np.allclose(mean[:, 0], [2, 5]) and np.allclose(rstd[:, 0], [0.5, 3.0 ** -0.5])
    assert np.allclose(y, [[-0.5, 6.0], [0.5, 1.0]])


def test_norm_of_groups_is_the_norm_of_each():
    rng = np.random.default_rng(0)
    x, w, b = rng.standard_normal((5, 12)), rng.standard_normal(12), rng.standard_normal(12)
    y, mean, rstd = HO.layer_norm(x, w, b, groups=3)
    for g in range(3):
        at = slice(4 * g, 4 * g + 4)
        yg, mg, rg = HO.layer_norm(x[:, at], w[at], b[at])
        assert np.allclose(y[:, at], yg) and np.allclose(mean[:, g], mg[:, 0]) and np.allclose(rstd[:, g], rg[:, 0])


def differences(f, x, d, h=1e-5):
    return (f(x + h * d) - f(x - h * d)) / (2 * h)


@pytest.mark.parametrize("groups", [1, 4])
def test_norm_gradients_against_differences(groups):
    rng = np.random.default_rng(1)
    x, w, b, dy = rng.standard_normal((6, 20)), rng.standard_normal(20), rng.standard_normal(20), rng.standard_normal((6, 20))
    dx, dw, db = HO.layer_norm_backward(dy, x, w, groups=groups)
    L = lambda x, w, b: (HO.layer_norm(x, w, b, groups=groups)[0] * dy).sum()
    d = rng.standard_normal(x.shape)
    assert np.isclose((dx * d).sum(), differences(lambda a: L(a, w, b), x, d), rtol=1e-7)
    d = rng.standard_normal(20)
    assert np.isclose((dw * d).sum(), differences(lambda a: L(x, a, b), w, d), rtol=1e-7)
    assert np.isclose((db * d).sum(), differences(lambda a: L(x, w, a), b, d), rtol=1e-7)


def test_attention_two_tokens_by_hand():
    # one head of one channel: S0 = 2, w = ln 2, u = 3; r = (1, 10), k = (4, 5), v = (6, 7)
    a = lambda *v: np.array(v, dtype=np.float64).reshape(-1, 1, 1)
    out, S = HO.attention(a(1, 10), a(4, 5), a(6, 7), np.array([np.log(2.0)]), np.array([[3.0]]), np.array([[[2.0]]]))
    # out_1 = 1 (2 + 3 * 24); S_1 = 1 + 24; out_2 = 10 (25 + 3 * 35); S_2 = 12.5 + 35
    assert np.allclose(out.ravel(), [74.0, 1300.0]) and np.allclose(S, 47.5)


def test_attention_is_the_numerator_of_wkv():
    """With one channel per head and k' = exp(k), the bonus exp(u) and r = 1, out / (out with v = 1) is Eq. "time mixing wkv"."""
    rng = np.random.default_rng(2)
    T, d = 9, 5
    k, v = rng.standard_normal((T, d)), rng.standard_normal((T, d))
    w, u = rng.uniform(0.1, 1.0, d), rng.standard_normal(d)
    one = np.ones((T, d, 1))
    run = lambda v: HO.attention(one, np.exp(k)[..., None], v[..., None], w, np.exp(u)[:, None])[0][..., 0]
    assert np.allclose(run(v) / run(np.ones_like(v)), BO.wkv_direct(k, v, w, u), rtol=1e-12)


def case(rng, T, H=3, D=4):
    r, k, v, do = (rng.standard_normal((T, H, D)) for _ in range(4))
    return r, k, v, do, np.exp(rng.uniform(-4, 0.5, H)), rng.standard_normal((H, D)), rng.standard_normal((H, D, D)), rng.standard_normal((H, D, D))


def test_sums_equal_the_recurrence_and_sequences_can_be_cut():
    rng = np.random.default_rng(3)
    r, k, v, _, w, u, S, _ = case(rng, 13)
    out, last = HO.attention(r, k, v, w, u, S)
    assert np.allclose(HO.attention_sums(r, k, v, w, u, S), out, rtol=1e-12)
    a, mid = HO.attention(r[:5], k[:5], v[:5], w, u, S)
    b, end = HO.attention(r[5:], k[5:], v[5:], w, u, mid)
    assert np.allclose(np.concatenate([a, b]), out, rtol=1e-13) and np.allclose(end, last, rtol=1e-13)


@pytest.mark.parametrize("T", [0, 1, 2, 11])
def test_attention_gradients_against_differences(T):
    rng = np.random.default_rng(4 + T)
    r, k, v, do, w, u, S, G = case(rng, T)

    def L(r, k, v, w, u, S):
        out, last = HO.attention(r, k, v, w, u, S)
        return (out * do).sum() + (last * G).sum()

    got = HO.attention_backward(r, k, v, do, w, u, S, G)
    args = [r, k, v, w, u, S]
    for i, g in enumerate(got):
        d = rng.standard_normal(args[i].shape)
        at = lambda a: L(*args[:i], a, *args[i + 1:])
        assert np.isclose((g * d).sum(), differences(at, args[i], d), rtol=1e-6, atol=1e-9), i
