"""GPU parity of the embedding lookup and its gradient with the oracle.

Bars.  Lookup: one product (2^-24) and half a step of the output's type.  Gradient: a row's terms are added one after the other, those of a
tile of sorted places and then the tiles, m additions in all, then a product and maybe an addition: (m + 2) 2^-24 of the sum of magnitudes."""
import numpy as np
import pytest

from oracle import tuning_oracle as TO
from paper_2505_03803_amd import binding as B

import gpu_util as G
from test_gpu_dropout import TYPES, half_step

pytestmark = pytest.mark.gpu
torch = G.torch_()


def ints(a):
    return torch.tensor(np.asarray(a), dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("T,vocab,d", [(1, 1, 1), (1, 50, 4096), (7, 9, 33), (300, 1000, 64), (65, 31, 1023), (5, 100, 5120), (3000, 17, 8)])
@pytest.mark.parametrize("tdt,odt", [("f16", "f16"), ("bf16", "bf16"), ("f32", "f32"), ("f32", "bf16"), ("f16", "f32"), ("bf16", "f16")])
def test_embedding(T, vocab, d, tdt, odt):
    rng = np.random.default_rng(T * 7 + d)
    torch.manual_seed(T + d)
    tokens = rng.integers(-1, vocab + 1, size=T)             # both ends outside the table
    table = torch.randn(vocab, d).to(TYPES[tdt]).cuda()
    scale = 1.0 if d % 2 else 1.7
    stride = d + (5 if T % 2 else 16)
    out = torch.full((T + 1, stride), 3.0, dtype=TYPES[odt], device="cuda")
    B.rwkvq_embedding(ints(tokens), T, table, B.DTYPES[tdt], vocab, d, scale, out, B.DTYPES[odt], out_stride=stride)
    want = torch.from_numpy(TO.embedding(tokens, table.cpu().double().numpy(), np.float32(scale).item()))
    got = out.cpu()
    assert bool(((got[:T, :d].double() - want).abs() <= half_step(TYPES[odt], want) + 2.0 ** -24 * want.abs()).all())
    assert bool((got[T] == 3.0).all()) and bool((got[:, d:] == 3.0).all())
    if scale == 1.0 and tdt == odt:
        assert torch.equal(got[:T, :d].double(), want)


# tokens of one row only, of few, of many; one, two and many tiles of sorted places; more than the 8192 that are sorted at once
SPREADS = {"same": lambda rng, T, V: np.full(T, V // 2), "few": lambda rng, T, V: rng.integers(0, min(V, 3), size=T),
           "even": lambda rng, T, V: rng.integers(0, V, size=T), "zipf": lambda rng, T, V: (np.exp(rng.random(T) * np.log(V + 1)) - 1).astype(int),
           "padded": lambda rng, T, V: np.where(rng.random(T) < 0.3, -1, rng.integers(0, V + 2, size=T)),
           "none": lambda rng, T, V: np.full(T, -1), "down": lambda rng, T, V: np.arange(T)[::-1] % V}
SIZES = [(1, 5, 8), (2, 1, 1), (31, 40, 24), (32, 7, 512), (33, 40, 520), (64, 100, 3), (65, 300, 1023), (777, 50, 64), (2048, 900, 40)]


def check_gradient(tokens, T, V, d, dt, scale, added, stride=None):
    t = TYPES[dt]
    stride = stride or d
    dout = torch.randn(T, stride).to(t).cuda()
    before = torch.randn(V, d).cuda() if added else torch.full((V, d), float("nan"), device="cuda")
    table = torch.full((V + 1, d), 5.0, device="cuda")       # and a row behind it
    table[:V] = before
    n = B.rwkvq_embedding_backward_workspace_size(T, d)
    ws = torch.full((n + 64,), 0x5A, dtype=torch.uint8, device="cuda")
    call = lambda: B.rwkvq_embedding_backward(ints(tokens), T, dout, B.DTYPES[dt], V, d, scale, table, added, ws, dout_stride=stride)  # noqa: E731
    call()
    got = table.clone()
    want, size, count = TO.embedding_backward(tokens, dout.cpu().double().numpy()[:, :d], V, np.float32(scale).item())
    old = before.cpu().double().numpy() if added else 0.0
    bar = 2.0 ** -24 * (count[:, None] + 2) * (size + np.abs(old)) + 2.0 ** -126
    err = np.abs(got[:V].cpu().double().numpy() - want - old)
    assert not (~(err <= bar)).any(), (np.argwhere(~(err <= bar))[:4], float(np.nanmax(err / bar)))
    assert bool((got[V] == 5.0).all()) and bool((ws[n:] == 0x5A).all())
    if added:
        assert torch.equal(got[:V][torch.from_numpy(count == 0).cuda()], before[torch.from_numpy(count == 0).cuda()])
    table[:V] = before
    ws.fill_(0xA5)
    call()
    assert torch.equal(got, table)


@pytest.mark.parametrize("T,V,d", SIZES)
@pytest.mark.parametrize("spread", sorted(SPREADS))
@pytest.mark.parametrize("added", [False, True])
def test_gradient(T, V, d, spread, added):
    rng = np.random.default_rng(T + V + d)
    torch.manual_seed(T + d)
    dt = ["f16", "bf16", "f32"][(T + len(spread)) % 3]
    check_gradient(SPREADS[spread](rng, T, V), T, V, d, dt, 1.0 if T % 2 else 0.3, added, d + (7 if d % 2 else 8))


# at the border between few tokens, taken without sorting, and more: 1024 of them, or 2048 pieces of 512 columns
@pytest.mark.parametrize("T,V,d", [(1024, 200, 1024), (1024, 90, 1025), (1025, 200, 33), (1025, 64, 512), (700, 50, 1501), (300, 40, 4096), (1024, 3, 3),
                                   (5, 40000, 72)])
@pytest.mark.parametrize("spread", ["same", "few", "zipf", "padded"])
@pytest.mark.parametrize("dt", ["f16", "bf16", "f32"])
def test_gradient_of_few_tokens(T, V, d, spread, dt):
    rng = np.random.default_rng(T + V + d)
    torch.manual_seed(T + d)
    check_gradient(SPREADS[spread](rng, T, V), T, V, d, dt, 0.3, dt == "bf16")


@pytest.mark.parametrize("T", [8192, 8193, 16384, 20011])
@pytest.mark.parametrize("spread", ["same", "zipf", "padded", "down"])
def test_gradient_of_many_tokens(T, spread):
    rng = np.random.default_rng(T)
    torch.manual_seed(T)
    check_gradient(SPREADS[spread](rng, T, 700), T, 700, 16, "f32", 1.0, spread == "zipf")


def test_infinities_stay_in_their_rows():
    T, V, d = 100, 9, 40
    tokens = np.arange(T) % V
    dout = torch.randn(T, d, device="cuda")
    dout[4] = float("inf")
    dout[13] = -float("inf")
    dout[5] = float("nan")
    tokens[20], tokens[21] = -1, V
    dout[20] = dout[21] = float("nan")                       # not read
    table = torch.empty(V, d, device="cuda")
    ws = torch.empty(B.rwkvq_embedding_backward_workspace_size(T, d), dtype=torch.uint8, device="cuda")
    B.rwkvq_embedding_backward(ints(tokens), T, dout, B.F32, V, d, 1.0, table, False, ws)
    bad = torch.isfinite(table).all(1).cpu()
    assert bad.tolist() == [v not in (4, 5) for v in range(V)] and bool(torch.isnan(table[4]).all())


def test_captured_and_replayed():
    T, V, d = 500, 60, 48
    rng = np.random.default_rng(0)
    tokens, dout, table = ints(rng.integers(0, V, size=T)), torch.randn(T, d, device="cuda"), torch.empty(V, d, device="cuda")
    ws = torch.empty(B.rwkvq_embedding_backward_workspace_size(T, d), dtype=torch.uint8, device="cuda")
    call = lambda to, w: B.rwkvq_embedding_backward(tokens, T, dout, B.F32, V, d, 1.0, to, False, w)  # noqa: E731
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call(table, ws)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(table, ws)
    for i in range(3):
        tokens.copy_(ints(rng.integers(-1, V if i else 2, size=T)))
        dout.normal_()
        graph.replay()
        want, other = torch.empty_like(table), torch.empty_like(ws)
        call(want, other)
        torch.cuda.synchronize()
        assert torch.equal(table, want)


def test_places_beyond_32_bits():
    """A table of 2^32 elements and more, rows of the output 2^27 apart; a gradient of as many."""
    V, d, T, far = 66000, 65536, 40, 1 << 27
    rng = np.random.default_rng(1)
    tokens = rng.integers(0, V, size=T)
    tokens[:3] = V - 1, 0, V - 1
    rows = torch.randn(T, d).to(torch.bfloat16).cuda()
    rows[2] = rows[0]
    table = torch.empty(V, d, dtype=torch.bfloat16, device="cuda")
    table[ints(tokens).long()] = rows
    out = torch.empty((T - 1) * far + d, dtype=torch.bfloat16, device="cuda")
    B.rwkvq_embedding(ints(tokens), T, table, B.BF16, V, d, 1.0, out, B.BF16, out_stride=far)
    placed = out.as_strided((T, d), (far, 1))
    assert torch.equal(placed, table[ints(tokens).long()])
    del table
    ws = torch.empty(B.rwkvq_embedding_backward_workspace_size(T, d), dtype=torch.uint8, device="cuda")
    grad = torch.full((V, d), float("nan"), device="cuda")
    B.rwkvq_embedding_backward(ints(tokens), T, out, B.BF16, V, d, 1.0, grad, False, ws, dout_stride=far)
    want = torch.zeros(T, d, dtype=torch.float64)
    for t in range(T):
        want[t] = sum(placed[i].double().cpu() for i in range(T) if tokens[i] == tokens[t])
    got = grad[ints(tokens).long()].cpu().double()
    assert bool(((got - want).abs() <= T * 2.0 ** -24 * want.abs().max()).all())
    grad[ints(tokens).long()] = 0.0
    assert not bool(grad.view(-1)[:1 << 32].any()) and not bool(grad.view(-1)[1 << 32:].any())


def test_many_tokens_of_a_training_step():
    rng = np.random.default_rng(2)
    torch.manual_seed(3)
    for dt in ("f16", "bf16"):
        check_gradient(SPREADS["zipf"](rng, 9000, 900), 9000, 900, 264, dt, 1.0, dt == "f16", 272)
