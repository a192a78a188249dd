"""CPU-side checks of tables whose matrices are not the adapters that the rows describe: a kernel would read or write behind them."""
import pytest
import torch

from paper_2505_03803_amd import binding as B

N, K, M = 24, 40, 6
half = lambda *shape: torch.zeros(shape, dtype=torch.float16)  # noqa: E731
f32 = lambda *shape: torch.zeros(shape)  # noqa: E731


def tables(a, b, da=None, db=None):
    rest = dict(xs=[half(M, K)] * len(a), hs=[f32(M, 128)] * len(a))
    return (B.AdapterTable(a, b, rest["xs"], [half(M, N)] * len(a)),
            B.AdapterGradTable(a, b, rest["xs"], rest["hs"], [half(M, N)] * len(a), None, da or [f32(*t.shape) for t in a], db or [f32(*t.shape) for t in b]))


@pytest.mark.parametrize("n,rank", [(3, 16), (2, 8), (2, 24), (9, 8)])
def test_other_adapters_than_the_rows(n, rank):
    rows = B.AdapterRows(1, M, n, rank)
    forward, grads = tables([half(2, 16, K)] * 2, [half(2, N, 16)] * 2)
    with pytest.raises(AssertionError):
        B.rwkvq_adapters(rows, forward, B.F16, B.F16)
    with pytest.raises(AssertionError):
        B.rwkvq_adapters_backward_workspace_size(rows, grads)
    with pytest.raises(AssertionError):
        B.rwkvq_adapters_backward(rows, grads, B.F16, f32(64))


@pytest.mark.parametrize("a,b", [((2, 16, K), (2, N, 8)), ((2, 16, K), (1, N, 16)), ((1, 16, K), (2, N, 16)), ((16, K), (N, 16))])
def test_matrices_that_do_not_belong_together(a, b):
    with pytest.raises(AssertionError):
        tables([half(2, 16, K), half(*a)], [half(2, N, 16), half(*b)])


def test_matrices_of_different_ranks():
    with pytest.raises(AssertionError):
        tables([half(2, 16, K), half(2, 8, K)], [half(2, N, 16), half(2, N, 8)])


@pytest.mark.parametrize("da,db", [((1, 16, K), (2, N, 16)), ((2, 16, K), (2, N, 8))])
def test_gradients_of_another_size(da, db):
    with pytest.raises(AssertionError):
        tables([half(2, 16, K)], [half(2, N, 16)], [f32(*da)], [f32(*db)])


def test_the_first_of_a_pool():
    """Rows may describe fewer adapters than the matrices hold."""
    _, grads = tables([half(3, 16, K)], [half(3, N, 16)])
    assert B.rwkvq_adapters_backward_workspace_size(B.AdapterRows(1, M, 2, 16), grads) > 0
