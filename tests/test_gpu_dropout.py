"""GPU parity of dropout with the oracle: which elements stay is compared element for element.

Bar of those that do: the factor (2^-24 of the product), the sum with base (2^-24 of both), and half a step of the output's type."""
import numpy as np
import pytest

from oracle import tuning_oracle as TO
from paper_2505_03803_amd import binding as B

import gpu_util as G

pytestmark = pytest.mark.gpu
torch = G.torch_()
TYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}


def half_step(t, value):
    """Half a step of the type at a value, at least that of its subnormals."""
    info = torch.finfo(t)
    return torch.clamp(value.abs() * (info.eps / 2), min=info.tiny * info.eps / 2)


def seed_of(key, number):
    return torch.tensor([key, number], dtype=torch.int64, device="cuda")


def rows(M, n, stride, t, spread=1.0):
    return (torch.randn(M, stride) * spread).to(t).cuda()


# rows of less than a counter's eight columns, odd ones, whole ones, more threads than a launch has
SIZES = [(1, 1), (3, 7), (2, 8), (5, 9), (77, 33), (1, 4096), (9, 1000), (130, 264), (700, 3)]


@pytest.mark.parametrize("M,n", SIZES)
@pytest.mark.parametrize("dt", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("base", [False, True])
def test_dropout(M, n, dt, base):
    torch.manual_seed(M * 1000 + n)
    t, p, key, number = TYPES[dt], 0.3, -(2 ** 61) + 12345 * M, 2 ** 62 + n
    stride = n + (3 if (M + n) % 2 else 24)                 # rows that 16-byte loads cannot and can begin at
    x, y = rows(M, n, stride, t, 3.0), torch.full((M + 1, stride), 7.0, dtype=t, device="cuda")
    z = rows(M, n, stride, t) if base else None
    B.rwkvq_dropout(x, B.DTYPES[dt], M, n, seed_of(key, number), p, y, base=z, x_stride=stride, base_stride=stride, y_stride=stride)
    stays, factor = TO.keep((key, number), p, M, n)
    x64, b64 = x.cpu().double()[:, :n], z.cpu().double()[:, :n] if base else torch.zeros(M, n, dtype=torch.float64)
    stays = torch.from_numpy(stays)
    want = torch.where(stays, x64 * factor, 0.0) + b64
    got = y.cpu()
    bar = half_step(t, want) + 2.0 ** -24 * (2 * (x64 * factor).abs() + b64.abs())
    assert bool(((got[:M, :n].double() - want).abs() <= bar).all())
    assert torch.equal(got[:M, :n][~stays], z.cpu()[:, :n][~stays] if base else torch.zeros_like(got[:M, :n][~stays]))
    assert bool((got[M] == 7.0).all()) and bool((got[:, n:] == 7.0).all())


@pytest.mark.parametrize("p,share", [(0.0, 1.0), (1.0, 0.0), (1e-7, 1.0)])
def test_ends_of_p(p, share):
    x = torch.randn(5, 40, device="cuda")
    y = torch.empty_like(x)
    B.rwkvq_dropout(x, B.F32, 5, 40, seed_of(1, 2), p, y)
    assert torch.equal(y, x * share)


def test_large():
    """Rows beyond 2^16 and more items than threads, against the share that stays and a few rows of the oracle."""
    M, n, p = 70001, 120, 0.1
    x, y = torch.ones(M, n, dtype=torch.float16, device="cuda"), torch.empty(M, n, dtype=torch.float16, device="cuda")
    B.rwkvq_dropout(x, B.F16, M, n, seed_of(11, 13), p, y)
    assert abs(float((y != 0).double().mean()) - 0.9) < 5 * (0.09 / (M * n)) ** 0.5 + 2.0 ** -16
    for row in (0, 65535, 65536, M - 1):
        words = [TO.philox((b, row, 13, 0), (11, 0)) for b in range(n // 8)]
        numbers = np.array([w >> s & 0xFFFF for four in words for w in four for s in (0, 16)])
        assert np.array_equal(y[row].cpu().numpy() != 0, numbers >= TO.limit(p))


@pytest.mark.parametrize("dt", ["f16", "bf16", "f32"])
def test_in_place_gradient_and_what_is_dropped(dt):
    t = TYPES[dt]
    torch.manual_seed(3)
    x = torch.randn(33, 64).to(t).cuda()
    s = seed_of(5, 6)
    y, z = torch.empty_like(x), x.clone()
    B.rwkvq_dropout(x, B.DTYPES[dt], 33, 64, s, 0.5, y)
    B.rwkvq_dropout(z, B.DTYPES[dt], 33, 64, s, 0.5, z)
    assert torch.equal(y, z)
    stays = torch.from_numpy(TO.keep((5, 6), 0.5, 33, 64)[0]).cuda()
    # an infinity or NaN that is dropped is gone
    bad = torch.where(stays, x, torch.full_like(x, float("nan")))
    bad[0][~stays[0]] = float("inf")
    B.rwkvq_dropout(bad, B.DTYPES[dt], 33, 64, s, 0.5, z)
    assert torch.equal(y, z)
    # added to itself
    B.rwkvq_dropout(x, B.DTYPES[dt], 33, 64, s, 0.5, z, base=x)
    w = x.clone()
    B.rwkvq_dropout(x, B.DTYPES[dt], 33, 64, s, 0.5, w, base=w)
    assert torch.equal(z, w)
    # the gradient: <dropout(x), dy> = <x, dropout(dy)>; p = 1/2 doubles exactly, so both sums have the same terms
    dy = torch.randn(33, 64).to(t).cuda()
    dx = torch.empty_like(dy)
    B.rwkvq_dropout(dy, B.DTYPES[dt], 33, 64, s, 0.5, dx)
    assert torch.equal(y.double() * dy.double(), x.double() * dx.double())


def test_graph_reads_the_seed_when_it_runs():
    x, y = torch.randn(40, 72, device="cuda"), torch.empty(40, 72, device="cuda")
    s = seed_of(1, 0)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        B.rwkvq_dropout(x, B.F32, 40, 72, s, 0.2, y)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.rwkvq_dropout(x, B.F32, 40, 72, s, 0.2, y)
    for number in (5, 6, 2 ** 40):
        s[1] = number
        graph.replay()
        want = torch.empty_like(y)
        got = y.clone()
        B.rwkvq_dropout(x, B.F32, 40, 72, s, 0.2, want)
        torch.cuda.synchronize()
        assert torch.equal(got, want) and np.array_equal((got != 0).cpu().numpy(), TO.keep((1, number), 0.2, 40, 72)[0])


def test_places_beyond_32_bits():
    far, M, n, p = 1 << 27, 40, 520, 0.3
    x, y = torch.randn(M, n, device="cuda").half(), torch.empty(M, n, dtype=torch.float16, device="cuda")
    wide, out = (torch.empty((M - 1) * far + n, dtype=torch.float16, device="cuda") for _ in range(2))
    wide.as_strided((M, n), (far, 1)).copy_(x)
    B.rwkvq_dropout(x, B.F16, M, n, seed_of(3, 2 ** 32 - 1), p, y)
    B.rwkvq_dropout(wide, B.F16, M, n, seed_of(3, 2 ** 32 - 1), p, out, x_stride=far, y_stride=far)
    assert torch.equal(out.as_strided((M, n), (far, 1)), y)
