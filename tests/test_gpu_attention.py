"""GPU parity of linear attention (prompts, single tokens, ragged batches) and its gradients with the binary64 oracle.

Bars.  Let A be a result of the oracle's formula with every term replaced by its magnitude.  A computed operand that meets the
matrix cores is held to 17 bits or more (2^-17 of it), at most two to a product; every sum is binary32, and on the way of a term
to a result there are at most T + 256 additions of 2^-24 (the recurrence token by token; far fewer where tokens are taken
together); exp(-x) of a binary32 product is off by (x + 2) 2^-24 of itself, which is below 2^-19 of the largest weight.  So a
16-bit result is within half an ulp + (2^-15 + (T + 256) 2^-24) A; states and the gradient of u, whose operands are held to 24
bits, within (T + 256 + 64) 2^-24 A; the gradient of w, which sums 17-bit products, as the 16-bit results without the half ulp."""
import numpy as np
import pytest

from oracle import heads_oracle as HO
from oracle import rwkvq_oracle as orc
from paper_2505_03803_amd import binding as B
from paper_2505_03803_amd import synth

import gpu_util as G

pytestmark = pytest.mark.gpu
HALF_ULP = {"f16": 2.0 ** -11, "bf16": 2.0 ** -8}
FLOOR = {"f16": 2.0 ** -25, "bf16": 2.0 ** -126}
NARROW = {"f16": synth.f32_to_f16_bits, "bf16": synth.f32_to_bf16_bits}
SENTINEL = 0x1234


def widen(bits, dt):
    return orc.widen(bits, dt).astype(np.float64)


def dev(a):
    a = np.ascontiguousarray(a)
    return G.torch_().from_numpy(a.view(np.int16) if a.dtype == np.uint16 else a).cuda()


def check(got, want, tol, what=""):
    bad = ~(np.abs(got - want) <= tol)
    assert not bad.any(), (what, int(bad.sum()), float(np.nanmax(np.abs(got - want) / np.maximum(tol, 1e-300))), np.argwhere(bad)[:4])


class Case:
    """Sequences of given lengths, `gap` rows in front of the first and behind the last one; slots: places in a larger pool."""

    def __init__(self, lens, H, D, dt, seed=0, offsets=True, slots=None, n_slots=0, gap=0, pad=0, w=None, scale=1.0, state=True):
        rng = np.random.default_rng(seed)
        self.lens, self.H, self.D, self.dt = lens, H, D, dt
        self.starts = [gap + sum(lens[:i]) for i in range(len(lens) + 1)]
        self.N = sum(lens) + 2 * gap
        self.wide, self.stride = H * D, H * D + pad
        self.bits = {p: NARROW[dt]((rng.standard_normal((self.N, self.stride)) * f * scale).astype(np.float32))
                     for p, f in (("r", 1.0), ("k", 0.5), ("v", 1.0), ("dout", 1.0))}
        self.x = {p: widen(b[:, :self.wide], dt).reshape(self.N, H, D) for p, b in self.bits.items()}
        self.w = (np.exp(rng.uniform(-5, 1, H)) if w is None else np.broadcast_to(np.asarray(w, dtype=np.float64), (H,))).astype(np.float32)
        self.u = (0.5 * rng.standard_normal((H, D))).astype(np.float32)
        self.slots = list(range(len(lens))) if slots is None else slots
        pool = n_slots or len(lens)
        self.S = (rng.standard_normal((pool, H, D, D)) * scale * scale).astype(np.float32) if state else None
        self.dS = (0.1 * rng.standard_normal((pool, H, D, D)) * scale).astype(np.float32)
        self.pool = pool
        self.d = {p: dev(b) for p, b in self.bits.items()}
        self.dw_, self.du_ = dev(self.w), dev(self.u)
        self.dS_in = None if self.S is None else dev(self.S)
        off = dev(np.array(self.starts, dtype=np.int32)) if offsets else None
        sl = None if slots is None else dev(np.array(slots, dtype=np.int32))
        self.heads = B.Heads(len(lens), self.N, H, D, offsets=off, slots=sl, n_slots=n_slots, r_stride=self.stride, k_stride=self.stride,
                             v_stride=self.stride, out_stride=self.stride)

    def forward(self, state_out=None):
        torch = G.torch_()
        out = torch.full((self.N, self.stride), SENTINEL, dtype=torch.int16, device="cuda")
        ws = torch.empty(max(B.rwkvq_linear_attention_workspace_size(self.heads), 16), dtype=torch.uint8, device="cuda")
        B.rwkvq_linear_attention(self.heads, self.d["r"], self.d["k"], self.d["v"], B.DTYPES[self.dt], self.dw_, self.du_, self.dS_in,
                                 state_out, out, ws)
        torch.cuda.synchronize()
        return out.cpu().numpy().view(np.uint16)

    def live(self):
        return [(b, s) for b, s in enumerate(self.slots) if 0 <= s < self.pool]

    def rows(self, b):
        return slice(self.starts[b], self.starts[b + 1])

    def check_untouched(self, bits):
        keep = np.ones(bits.shape, dtype=bool)
        for b, _ in self.live():
            keep[self.rows(b), :self.wide] = False
        assert np.all(bits[keep] == SENTINEL)

    def check_forward(self):
        torch = G.torch_()
        so = torch.full((self.pool, self.H, self.D, self.D), 7.0, device="cuda")
        bits = self.forward(so)
        self.check_untouched(bits)
        got, so = widen(bits[:, :self.wide], self.dt).reshape(self.N, self.H, self.D), so.cpu().numpy().astype(np.float64)
        seen = set()
        for b, s in self.live():
            at = self.rows(b)
            S = None if self.S is None else self.S[s]
            args = [self.x[p][at] for p in "rkv"]
            want, last = HO.attention(*args, self.w, self.u, S)
            A, lastA = HO.attention(*[np.abs(a) for a in args], self.w, np.abs(self.u), None if S is None else np.abs(S))
            e = (self.lens[b] + 256) * 2.0 ** -24
            check(got[at], want, HALF_ULP[self.dt] * 1.01 * np.abs(want) + FLOOR[self.dt] + (2.0 ** -15 + e) * A, f"out {b}")
            check(so[s], last, (e + 64 * 2.0 ** -24) * lastA, f"state {b}")
            seen.add(s)
        for s in range(self.pool):
            assert s in seen or np.all(so[s] == 7.0)
        return bits

    def backward(self, dstate=True):
        torch = G.torch_()
        full = lambda: torch.full((self.N, self.stride), SENTINEL, dtype=torch.int16, device="cuda")
        o = dict(dr=full(), dk=full(), dv=full(), dw=torch.full((self.H + 1,), 7.0, device="cuda"),
                 du=torch.full((self.H * self.D + 1,), 7.0, device="cuda"), di=torch.full((self.pool, self.H, self.D, self.D), 7.0, device="cuda"))
        ws = torch.empty(max(B.rwkvq_linear_attention_backward_workspace_size(self.heads), 16), dtype=torch.uint8, device="cuda")
        B.rwkvq_linear_attention_backward(self.heads, self.d["r"], self.d["k"], self.d["v"], self.d["dout"], B.DTYPES[self.dt], self.dw_, self.du_,
                                          self.dS_in, dev(self.dS) if dstate else None, o["dr"], o["dk"], o["dv"], o["dw"], o["du"], o["di"], ws)
        torch.cuda.synchronize()
        return {p: t.cpu().numpy() for p, t in o.items()}

    def check_backward(self, dstate=True):
        o = self.backward(dstate)
        want_w, A_w, want_u, A_u = (np.zeros(s) for s in ((self.H,), (self.H,), (self.H, self.D), (self.H, self.D)))
        seen = set()
        for p in ("dr", "dk", "dv"):
            self.check_untouched(o[p].view(np.uint16))
        for b, s in self.live():
            at = self.rows(b)
            S, G_ = None if self.S is None else self.S[s], self.dS[s] if dstate else None
            args = [self.x[p][at] for p in ("r", "k", "v", "dout")]
            want = HO.attention_backward(*args, self.w, self.u, S, G_)
            A = HO.attention_backward(*[np.abs(a) for a in args], self.w, np.abs(self.u), None if S is None else np.abs(S),
                                      None if G_ is None else np.abs(G_))
            e = (self.lens[b] + 256) * 2.0 ** -24
            for p, x, a in zip(("dr", "dk", "dv"), want, A):
                got = widen(o[p].view(np.uint16)[at, :self.wide], self.dt).reshape(-1, self.H, self.D)
                check(got, x, HALF_ULP[self.dt] * 1.01 * np.abs(x) + FLOOR[self.dt] + (2.0 ** -15 + e) * a, f"{p} {b}")
            check(o["di"][s].astype(np.float64), want[5], (e + 64 * 2.0 ** -24) * A[5], f"dstate_in {b}")
            want_w += want[3]; A_w += np.abs(A[3]); want_u += want[4]; A_u += A[4]
            seen.add(s)
        e = (self.N + 256) * 2.0 ** -24
        check(o["dw"][:-1].astype(np.float64), want_w, (2.0 ** -15 + e) * A_w, "dw")
        check(o["du"][:-1].astype(np.float64).reshape(self.H, self.D), want_u, (e + 64 * 2.0 ** -24) * A_u, "du")
        assert o["dw"][-1] == 7.0 and o["du"][-1] == 7.0
        for s in range(self.pool):
            assert s in seen or np.all(o["di"][s] == 7.0)


DIMS = [(3, 8), (2, 16), (5, 24), (3, 32), (2, 40), (4, 64), (2, 72), (3, 80), (2, 104), (2, 128)]


@pytest.mark.parametrize("H,D", DIMS)
@pytest.mark.parametrize("dt", ["f16", "bf16"])
def test_head_dims(H, D, dt):
    print(f"attention H={H} D={D} {dt}", flush=True)
    c = Case([70, 1, 133], H, D, dt, seed=D, pad=8)
    c.check_forward()
    c.check_backward()


@pytest.mark.parametrize("T", [1, 2, 3, 15, 16, 17, 31, 32, 33, 63, 64, 65, 100, 127, 128, 129, 191, 192, 193, 257, 320, 500, 777])
@pytest.mark.parametrize("dt", ["f16", "bf16"])
def test_lengths(T, dt):
    print(f"attention T={T} {dt}", flush=True)
    c = Case([T], 2, 64, dt, seed=T, offsets=False)
    c.check_forward()
    c.check_backward()


@pytest.mark.parametrize("B_,T,H,D", [(2, 65, 3, 32), (7, 64, 2, 64), (3, 200, 2, 128), (9, 1, 5, 64), (300, 1, 2, 64), (1, 1, 64, 64), (4, 1, 3, 128),
                                      (33, 1, 2, 40), (65, 2, 1, 64), (40, 130, 8, 64), (5, 1, 1, 8)])
def test_equal_lengths(B_, T, H, D):
    print(f"attention B={B_} T={T} H={H} D={D}", flush=True)
    c = Case([T] * B_, H, D, "bf16", seed=B_ + T, offsets=False)
    c.check_forward()
    c.check_backward()


@pytest.mark.parametrize("lens", [[0], [0, 0, 5], [5, 0, 0], [1, 0, 64, 65, 0, 300, 1, 1], [1] * 20, [0] * 9 + [400], [129, 3, 64, 1, 0, 2, 200]])
@pytest.mark.parametrize("dt,H,D", [("f16", 2, 64), ("bf16", 3, 40), ("bf16", 2, 128)])
def test_ragged_and_empty_sequences(lens, dt, H, D):
    print(f"attention lens={lens} {dt} D={D}", flush=True)
    c = Case(lens, H, D, dt, seed=len(lens), gap=3, pad=16)
    c.check_forward()
    c.check_backward()


@pytest.mark.parametrize("lens", [[1, 1, 1, 1, 1], [70, 0, 130, 1, 40], [1, 200, 3, 65, 64]])
def test_slots(lens):
    """Sequences in a pool of nine slots; those whose slot is none of it are left out."""
    for slots in ([8, 0, 3, 5, 2], [4, -1, 7, 9, 0], [-5, 100, 2 ** 31 - 1, 9, -1]):
        print(f"attention lens={lens} slots={slots}", flush=True)
        for offsets in ([True, False] if len(set(lens)) == 1 else [True]):
            c = Case(lens, 2, 64, "bf16", seed=7, slots=slots, n_slots=9, offsets=offsets)
            c.check_forward()
            c.check_backward()


@pytest.mark.parametrize("w", [0.0, 1e-6, 0.3, 5.0, 90.0, 1e4, -0.02])
def test_decays(w):
    """From heads that forget nothing to heads that forget at once, and a state that grows."""
    print(f"attention w={w}", flush=True)
    c = Case([150, 66], 2, 64, "bf16", seed=3, w=w)
    c.check_forward()
    c.check_backward()


@pytest.mark.parametrize("dt,scale", [("f16", 30.0), ("f16", 1e-3), ("bf16", 1e6), ("bf16", 1e-6)])
def test_magnitudes(dt, scale):
    """Scores and states beyond fp16's range and far below it."""
    c = Case([130], 2, 64, dt, seed=4, scale=scale)
    if dt == "f16" and scale > 1:
        c.bits["r"] = NARROW[dt]((c.x["r"].reshape(c.N, -1) / scale / scale / scale).astype(np.float32))     # outputs that fp16 holds
        c.x["r"], c.d["r"] = widen(c.bits["r"], dt).reshape(c.N, c.H, c.D), dev(c.bits["r"])
    c.check_forward()
    if dt == "bf16":
        c.dS *= np.float32(scale)
        c.check_backward()


def test_without_states():
    c = Case([90, 1, 64], 3, 64, "f16", seed=5, state=False)
    c.check_forward()
    c.check_backward(dstate=False)
    assert np.array_equal(c.forward(None), c.forward(None))


def test_state_in_place_token_by_token():
    """Single tokens with the state in place, then in chunks: each against the oracle's whole sequence."""
    torch = G.torch_()
    T, H, D = 21, 3, 64
    c = Case([T], H, D, "bf16", seed=6, offsets=False)
    want, last = HO.attention(c.x["r"], c.x["k"], c.x["v"], c.w, c.u, c.S[0])
    A, lastA = HO.attention(*[np.abs(c.x[p]) for p in "rkv"], c.w, np.abs(c.u), np.abs(c.S[0]))
    e = (T + 256) * 2.0 ** -24
    for cuts in (list(range(T + 1)), [0, 1, 8, 9, 21], [0, 20, 21]):
        state = dev(c.S)
        out = torch.empty((T, H * D), dtype=torch.int16, device="cuda")
        for a, b in zip(cuts, cuts[1:]):
            h = B.Heads(1, b - a, H, D)
            ws = torch.empty(max(B.rwkvq_linear_attention_workspace_size(h), 16), dtype=torch.uint8, device="cuda")
            B.rwkvq_linear_attention(h, c.d["r"][a:b], c.d["k"][a:b], c.d["v"][a:b], B.BF16, c.dw_, c.du_, state, state, out[a:b], ws)
        torch.cuda.synchronize()
        got = widen(out.cpu().numpy().view(np.uint16), "bf16").reshape(T, H, D)
        check(got, want, HALF_ULP["bf16"] * 1.01 * np.abs(want) + (2.0 ** -15 + e) * A, str(cuts))
        check(state.cpu().numpy()[0].astype(np.float64), last, (e + 64 * 2.0 ** -24) * lastA, str(cuts))


def test_offsets_out_of_order_stay_inside():
    """Offsets that no caller should give are limited to the rows there are: neighbours of the buffers keep their values."""
    torch = G.torch_()
    c = Case([40, 40, 40], 2, 64, "f16", seed=8)
    bad = torch.tensor([-7, 55, 20, 2 ** 31 - 1], dtype=torch.int32, device="cuda")
    c.heads = B.Heads(3, 120, 2, 64, offsets=bad)
    hold = torch.full((200, 128), SENTINEL, dtype=torch.int16, device="cuda")
    ws = torch.empty(max(B.rwkvq_linear_attention_workspace_size(c.heads), 16), dtype=torch.uint8, device="cuda")
    B.rwkvq_linear_attention(c.heads, c.d["r"], c.d["k"], c.d["v"], B.F16, c.dw_, c.du_, c.dS_in, None, hold[40:160], ws)
    torch.cuda.synchronize()
    assert bool((hold[:40] == SENTINEL).all()) and bool((hold[160:] == SENTINEL).all())


def test_rows_beyond_32_bits():
    """Rows that begin more than 2^31 elements behind the first: r, k, v and out are columns of one wide buffer."""
    torch = G.torch_()
    T, H, D, stride = 131, 1, 64, 1 << 24
    c = Case([T], H, D, "bf16", seed=9, offsets=False)
    buf = torch.empty(stride * (T - 1) + 8 * D, dtype=torch.int16, device="cuda")
    view = lambda i: torch.as_strided(buf, (T, D), (stride, 1), i * D)
    for i, p in enumerate(("r", "k", "v", "dout")):
        view(i).copy_(c.d[p])
    h = B.Heads(1, T, H, D, r_stride=stride, k_stride=stride, v_stride=stride, out_stride=stride)
    so = torch.empty((1, H, D, D), device="cuda")
    ws = torch.empty(max(B.rwkvq_linear_attention_workspace_size(h), B.rwkvq_linear_attention_backward_workspace_size(h), 16), dtype=torch.uint8, device="cuda")
    B.rwkvq_linear_attention(h, view(0), view(1), view(2), B.BF16, c.dw_, c.du_, c.dS_in, so, view(4), ws)
    torch.cuda.synchronize()
    assert np.array_equal(view(4).cpu().numpy().view(np.uint16), c.forward(None))
    dw, du, di = torch.empty(H, device="cuda"), torch.empty((H, D), device="cuda"), torch.empty_like(so)
    B.rwkvq_linear_attention_backward(h, view(0), view(1), view(2), view(3), B.BF16, c.dw_, c.du_, c.dS_in, dev(c.dS), view(5), view(6), view(7), dw, du, di, ws)
    torch.cuda.synchronize()
    o = c.backward()
    for i, p in enumerate(("dr", "dk", "dv")):
        assert np.array_equal(view(5 + i).cpu().numpy(), o[p])
    assert np.array_equal(dw.cpu().numpy(), o["dw"][:-1])
    del buf
    torch.cuda.empty_cache()


@pytest.mark.parametrize("lens,H", [([64], 2), ([1, 1, 1], 4), ([300, 20, 1, 129], 2), ([1500], 4)])
def test_same_bits_again_on_another_stream_and_in_a_graph(lens, H):
    torch = G.torch_()
    c = Case(lens, H, 64, "bf16", seed=10, offsets=len(set(lens)) > 1)
    out, so = torch.empty((c.N, c.wide), dtype=torch.int16, device="cuda"), torch.empty_like(c.dS_in)
    dr, dk, dv = (torch.empty_like(out) for _ in range(3))
    dw, du, di = torch.empty(H, device="cuda"), torch.empty((H, 64), device="cuda"), torch.empty_like(so)
    ws = torch.empty(max(B.rwkvq_linear_attention_workspace_size(c.heads), 16), dtype=torch.uint8, device="cuda")
    wb = torch.empty(B.rwkvq_linear_attention_backward_workspace_size(c.heads), dtype=torch.uint8, device="cuda")
    dS = dev(c.dS)

    def both():
        B.rwkvq_linear_attention(c.heads, c.d["r"], c.d["k"], c.d["v"], B.BF16, c.dw_, c.du_, c.dS_in, so, out, ws)
        B.rwkvq_linear_attention_backward(c.heads, c.d["r"], c.d["k"], c.d["v"], c.d["dout"], B.BF16, c.dw_, c.du_, c.dS_in, dS, dr, dk, dv, dw, du, di, wb)

    outs = [out, so, dr, dk, dv, dw, du, di]
    both()
    torch.cuda.synchronize()
    first = [t.clone() for t in outs]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        both()
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(first, outs))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        both()
    for _ in range(3):
        c.d["v"].copy_(c.d["v"].roll(1, 1)); c.dS_in.mul_(0.5)
        for t in outs:
            t.zero_()
        g.replay()
        torch.cuda.synchronize()
        replayed = [t.clone() for t in outs]
        both()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(replayed, outs))


def test_gradients_against_differences():
    """<gradient, direction> against the central difference of the oracle's forward pass at the bf16 inputs.  The 16-bit
    gradients carry half an ulp (2^-8 of each product, with random signs: four standard deviations of their sum), dw and du
    2^-15 of the sum of their terms' magnitudes, which the directions weigh."""
    c = Case([83], 2, 64, "bf16", seed=11, offsets=False)
    o = c.backward()
    x = [c.x["r"], c.x["k"], c.x["v"], c.w.astype(np.float64), c.u.astype(np.float64), c.S[0].astype(np.float64)]

    def L(*a):
        out, last = HO.attention(*a)
        return (out * c.x["dout"]).sum() + (last * c.dS[0]).sum()

    rng = np.random.default_rng(12)
    got = [widen(o[p].view(np.uint16)[:, :c.wide], "bf16").reshape(c.N, c.H, c.D) for p in ("dr", "dk", "dv")]
    got += [o["dw"][:-1].astype(np.float64), o["du"][:-1].astype(np.float64).reshape(c.H, c.D), o["di"][0].astype(np.float64)]
    A = HO.attention_backward(*[np.abs(c.x[p]) for p in ("r", "k", "v", "dout")], c.w, np.abs(c.u), np.abs(c.S[0]), np.abs(c.dS[0]))
    for i, g in enumerate(got):
        d, h = rng.standard_normal(x[i].shape), 1e-4
        want = (L(*x[:i], x[i] + h * d, *x[i + 1:]) - L(*x[:i], x[i] - h * d, *x[i + 1:])) / (2 * h)
        terms = g * d
        bar = 2.0 ** -15 * np.abs(A[i] * d).sum() + 1e-6 * abs(want) + (4 * 2.0 ** -8 * np.sqrt((terms ** 2).sum()) if i < 3 else 0.0)
        assert abs(terms.sum() - want) <= bar, (i, terms.sum(), want, bar)


@pytest.mark.parametrize("bad", ["inf", "nan"])
@pytest.mark.parametrize("dt,H,D,T,t0", [("f16", 2, 64, 150, 70), ("bf16", 2, 64, 150, 70), ("bf16", 3, 40, 90, 87), ("f16", 2, 24, 50, 0), ("f16", 2, 128, 150, 70),
                                         ("bf16", 2, 104, 70, 63), ("bf16", 2, 64, 300, 64)])
def test_infinities_reach_only_what_they_should(dt, H, D, T, t0, bad):
    """One infinity or NaN in r, k, v or dout of token t0, head 1, channel c: what the formulas make of it is not finite, and every other
    number keeps its bits (earlier tokens of the same chunk among them)."""
    print(f"attention {bad} in {dt} D={D} T={T}", flush=True)
    torch = G.torch_()
    w, c = [0.1] * H, D - 3
    value = {"f16": dict(inf=0x7C00, nan=0x7E00), "bf16": dict(inf=0xFF80, nan=0x7FC0)}[dt][bad]

    def run(case):
        so = torch.full((1, H, D, D), 7.0, device="cuda")
        got = dict(out=case.forward(so), so=so.cpu().numpy())
        got.update(case.backward())
        got["dw"], got["du"] = got["dw"][:-1], got["du"][:-1].reshape(H, D)
        return {p: widen(a.view(np.uint16), dt).reshape(T, H, D) if p in ("out", "dr", "dk", "dv") else a for p, a in got.items()}

    clean = run(Case([T], H, D, dt, seed=5, w=w, offsets=False))
    all_ = slice(None)
    reached = dict(                                # result: (tokens or none, channels)
        v=dict(out=(slice(t0, None), c), so=(all_, c), dr=(slice(t0, None), all_), dk=(t0, all_), du=(all_,), dw=()),
        k=dict(out=(slice(t0, None), all_), so=(c, all_), dr=(slice(t0, None), c), dv=(t0, all_), du=(c,), dw=()),
        r=dict(out=(t0, all_), di=(c, all_), dk=(slice(0, t0 + 1), c), dv=(slice(0, t0 + 1), all_), du=(c,), dw=()),
        dout=dict(di=(all_, c), dr=(t0, all_), dk=(slice(0, t0 + 1), all_), dv=(slice(0, t0 + 1), c), du=(all_,), dw=()))
    for p, where in reached.items():
        case = Case([T], H, D, dt, seed=5, w=w, offsets=False)
        case.bits[p][t0, D + c] = value
        case.d[p] = dev(case.bits[p])
        got = run(case)
        for name, a in got.items():
            want = np.zeros(a.shape, dtype=bool)
            if name in where:
                at = where[name]
                if name in ("out", "dr", "dk", "dv"):
                    want[at[0], 1, at[1]] = True
                elif name in ("so", "di"):
                    want[0, 1, at[0], at[1]] = True
                else:
                    want[(1, *at)] = True
            assert not np.isfinite(a[want]).any(), (p, name)
            assert np.array_equal(a[~want], clean[name][~want]), (p, name)


@pytest.mark.parametrize("lens,H,D,dt", [([2305], 1, 64, "bf16"), ([70, 2500, 0, 129], 2, 32, "f16"), ([2200, 1], 1, 128, "bf16"), ([2177], 1, 104, "f16")])
def test_long_sequences(lens, H, D, dt):
    """More segments than a workgroup adds up by itself."""
    print(f"attention lens={lens} D={D} {dt}", flush=True)
    c = Case(lens, H, D, dt, seed=sum(lens), w=[0.003, 0.3][:H], offsets=len(lens) > 1)
    c.check_forward()
    c.check_backward()


@pytest.mark.parametrize("dt,H,D,T", [("bf16", 2, 64, 150), ("f16", 2, 128, 70), ("f16", 2, 64, 1)])
def test_infinite_decay(dt, H, D, T):
    """A decay that leaves nothing: the same bits as one whose powers are 0, tokens in front still count with the weight 1."""
    torch = G.torch_()
    got = []
    for w in (1e4, np.inf):
        c = Case([T], H, D, dt, seed=11, w=[w, 0.5], offsets=False)
        so = torch.full((1, H, D, D), 7.0, device="cuda")
        got.append((c.forward(so), so.cpu().numpy(), c.backward()))
    assert np.array_equal(got[0][0], got[1][0]) and np.array_equal(got[0][1], got[1][1])
    assert all(np.array_equal(got[0][2][p], got[1][2][p]) for p in got[0][2])
