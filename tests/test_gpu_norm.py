"""GPU parity of layer norm and its gradients with the binary64 oracle.

Bars.  A sum of n terms over 256 threads or fewer rounds at most n / 64 + 32 times on any way from a term to the result, so it
is off by at most gamma = (n / 64 + 32) 2^-24 of the sum of magnitudes.  With z = max |x - mean| rstd and m = max |x| rstd per
group, xhat is off by 2 gamma (m + z) in all (mean, variance, the difference, the quotient), y by |weight| times that and two
roundings, plus half an output ulp; the gradients by the same with the magnitudes of their terms.  mean and rstd that the
backward pass reads are binary32 values: 2^-24 of them, within the same bar."""
import numpy as np
import pytest

from oracle import heads_oracle as HO
from oracle import rwkvq_oracle as orc
from paper_2505_03803_amd import binding as B
from paper_2505_03803_amd import synth

import gpu_util as G

pytestmark = pytest.mark.gpu
HALF_ULP = {"f16": 2.0 ** -11, "bf16": 2.0 ** -8, "f32": 2.0 ** -24}
FLOOR = {"f16": 2.0 ** -25, "bf16": 2.0 ** -126, "f32": 2.0 ** -126}
NARROW = {"f16": synth.f32_to_f16_bits, "bf16": synth.f32_to_bf16_bits, "f32": lambda a: np.ascontiguousarray(a, dtype=np.float32)}


def widen(a, dt):
    return a.astype(np.float64) if dt == "f32" else orc.widen(a, dt).astype(np.float64)


def rows(rng, M, width, stride, dt, spread=1.0, offset=0.0):
    """[M][stride] on the GPU, of which `width` columns count, and those in binary64."""
    a = NARROW[dt](rng.standard_normal((M, stride)).astype(np.float32) * spread + offset)
    dev = G.torch_().from_numpy(a if dt == "f32" else a.view(np.int16)).cuda()
    return dev, widen(a[:, :width], dt)


def host(t, dt):
    a = t.cpu().numpy()
    return a.astype(np.float64) if dt == "f32" else widen(a.view(np.uint16), dt)


def f32(a):
    return G.torch_().from_numpy(np.ascontiguousarray(a, dtype=np.float32)).cuda()


def wide32(t):
    return t.cpu().numpy().astype(np.float64)


def gamma(n):
    return (n / 64 + 32) * 2.0 ** -24


def check(got, want, tol):
    bad = ~(np.abs(got - want) <= tol)
    assert not bad.any(), (int(bad.sum()), float(np.nanmax(np.abs(got - want) / np.maximum(tol, 1e-300))), np.argwhere(bad)[:4])


def xhat_error(x, groups, eps):
    """The bar of xhat, [M][groups n]."""
    n = x.shape[1] // groups
    _, mean, rstd = HO.layer_norm(x, None, None, eps, groups)
    z = x.reshape(len(x), groups, n)
    big = (np.abs(z).max(-1) + np.abs(z - mean[..., None]).max(-1)) * rstd
    return np.repeat(2 * gamma(n) * big, n, axis=1)


# widths: one value, less than a 16-byte load, odd ones, one load per lane, several, a workgroup's worth, more than its registers hold
SIZES = [(1, 1, 1), (3, 1, 2), (5, 1, 7), (2, 1, 8), (4, 1, 63), (3, 1, 64), (5, 1, 65), (2, 1, 250), (7, 1, 256), (3, 1, 1000), (300, 1, 1023),
         (2, 1, 1024), (1, 1, 4096), (65, 1, 4096), (9, 1, 5120), (2, 1, 8192), (3, 1, 10001), (2, 1, 16384), (2, 1, 16392), (2, 1, 40003),
         (1, 64, 64), (33, 64, 64), (5, 3, 8), (7, 80, 64), (4, 5, 33), (3, 40, 128), (129, 2, 24), (2, 7, 1), (3, 2, 4104), (700, 16, 16)]


@pytest.mark.parametrize("M,groups,n", SIZES)
@pytest.mark.parametrize("dt", ["f16", "bf16", "f32"])
def test_norm(M, groups, n, dt):
    rng = np.random.default_rng(M * 100003 + groups * 1009 + n)
    wide = groups * n
    odd = (M + n) % 2
    stride = wide + (3 if odd else 16)                    # rows that 16-byte loads cannot and can begin at
    x, x64 = rows(rng, M, wide, stride, dt, 2.0, 0.7)
    w, b = rng.standard_normal(wide).astype(np.float32), rng.standard_normal(wide).astype(np.float32)
    eps = 1e-5
    print(f"norm M={M} groups={groups} n={n} {dt} stride={stride}", flush=True)
    torch = G.torch_()
    y = torch.full((M, wide + 8), 7, dtype=x.dtype, device="cuda")
    mean, rstd = (torch.empty((M, groups), dtype=torch.float32, device="cuda") for _ in range(2))
    B.rwkvq_layer_norm(x, B.DTYPES[dt], M, groups, n, f32(w), f32(b), eps, y, mean, rstd, x_stride=stride, y_stride=wide + 8)
    torch.cuda.synchronize()
    want, wm, wr = HO.layer_norm(x64, w, b, eps, groups)
    bar = xhat_error(x64, groups, eps) * np.abs(w) + 2.0 ** -23 * (np.abs(want) + np.abs(b))
    check(host(y[:, :wide].contiguous(), dt), want, bar + HALF_ULP[dt] * 1.01 * np.abs(want) + FLOOR[dt])
    assert bool((y[:, wide:] == 7).all())                 # nothing behind the rows
    z = x64.reshape(M, groups, n)
    check(wide32(mean), wm, gamma(n) * np.abs(z).max(-1) + 2.0 ** -126)
    # var is off by 2 gamma (|x| + |x - mean|) |x - mean| at most, and 1 / sqrt turns a relative error into half of it
    big = (np.abs(z).max(-1) + np.abs(z - wm[..., None]).max(-1)) * wr
    check(wide32(rstd), wr, wr * (2 * gamma(n) * (big + 1) * big + 2.0 ** -22))


@pytest.mark.parametrize("dt", ["f16", "bf16", "f32"])
def test_norm_without_weights_in_place_and_large_means(dt):
    rng = np.random.default_rng(5)
    x, x64 = rows(rng, 37, 512, 512, dt, 1.0, 100.0)
    B.rwkvq_layer_norm(x, B.DTYPES[dt], 37, 1, 512, None, None, 1e-6, x)
    want, _, _ = HO.layer_norm(x64, eps=1e-6)
    check(host(x, dt), want, xhat_error(x64, 1, 1e-6) + HALF_ULP[dt] * 1.01 * np.abs(want) + FLOOR[dt])


def test_norm_of_equal_values_is_the_bias():
    torch = G.torch_()
    x = torch.full((3, 96), 2.5, device="cuda")
    y = torch.empty_like(x)
    b = torch.arange(96, dtype=torch.float32, device="cuda")
    B.rwkvq_layer_norm(x, B.F32, 3, 1, 96, None, b, 1e-5, y)
    assert torch.equal(y, b.expand(3, -1))


@pytest.mark.parametrize("M,groups,n", SIZES + [(1500, 1, 512), (5000, 1, 40), (2111, 4, 64), (600, 1, 8192)])
@pytest.mark.parametrize("dt", ["f16", "bf16", "f32"])
def test_norm_backward(M, groups, n, dt):
    rng = np.random.default_rng(M * 100003 + groups * 1009 + n + 1)
    torch = G.torch_()
    wide, odd, eps = groups * n, (M + n) % 2, 1e-5
    xs, ds = wide + (0 if odd else 8), wide + (5 if odd else 24)
    x, x64 = rows(rng, M, wide, xs, dt, 1.5, -0.4)
    dy, dy64 = rows(rng, M, wide, ds, dt)
    w = rng.standard_normal(wide).astype(np.float32)
    _, mean, rstd = HO.layer_norm(x64, None, None, eps, groups)
    print(f"norm backward M={M} groups={groups} n={n} {dt}", flush=True)
    dx = torch.full((M, wide + 8), 7, dtype=x.dtype, device="cuda")
    dw, db = (torch.full((wide + 1,), 7.0, device="cuda") for _ in range(2))
    ws = torch.empty(B.rwkvq_layer_norm_backward_workspace_size(M, groups, n), dtype=torch.uint8, device="cuda")
    args = (x, B.DTYPES[dt], M, groups, n, f32(w), f32(mean), f32(rstd))
    more = dict(dy_stride=ds, x_stride=xs)
    B.rwkvq_layer_norm_backward(dy, *args, dx, dw, db, ws, dx_stride=wide + 8, **more)
    torch.cuda.synchronize()
    want_x, want_w, want_b = HO.layer_norm_backward(dy64, x64, w, eps, groups)
    e = xhat_error(x64, groups, eps)
    xhat, _, _ = HO.layer_norm(x64, None, None, eps, groups)
    shape = (M, groups, n)
    g, big = np.abs(dy64 * w).reshape(shape), (np.abs(xhat) + e).reshape(shape)
    each = e.reshape(shape)
    c2 = (g * big).mean(-1, keepdims=True)
    bar = rstd[..., None] * (4 * gamma(n) * (g + g.mean(-1, keepdims=True) + big * c2) + each * c2 + big * (g * each).mean(-1, keepdims=True))
    check(host(dx[:, :wide].contiguous(), dt), want_x, bar.reshape(M, wide) + HALF_ULP[dt] * 1.01 * np.abs(want_x) + FLOOR[dt])
    assert bool((dx[:, wide:] == 7).all()) and float(dw[-1]) == 7.0 and float(db[-1]) == 7.0
    sums = (M + 32) * 2.0 ** -24
    check(wide32(dw)[:wide], want_w, sums * (np.abs(dy64) * np.abs(xhat)).sum(0) + (np.abs(dy64) * e).sum(0) + 2.0 ** -126)
    check(wide32(db)[:wide], want_b, sums * np.abs(dy64).sum(0) + 2.0 ** -126)
    # the parts alone, and again: the same bits
    dx2, dw2, db2 = torch.full_like(dx, 7), torch.full_like(dw, 7.0), torch.full_like(db, 7.0)
    B.rwkvq_layer_norm_backward(dy, *args, dx2, None, None, ws, dx_stride=wide + 8, **more)
    B.rwkvq_layer_norm_backward(dy, *args, None, dw2, db2, ws, **more)
    again = torch.full_like(dw, 7.0)
    B.rwkvq_layer_norm_backward(dy, *args, None, again, torch.empty_like(db), ws, **more)
    torch.cuda.synchronize()
    check(host(dx2[:, :wide].contiguous(), dt), want_x, bar.reshape(M, wide) + HALF_ULP[dt] * 1.01 * np.abs(want_x) + FLOOR[dt])
    check(wide32(dw2)[:wide], want_w, sums * (np.abs(dy64) * np.abs(xhat)).sum(0) + (np.abs(dy64) * e).sum(0) + 2.0 ** -126)
    assert torch.equal(dw2, again)


def test_norm_backward_in_place_without_weight():
    rng = np.random.default_rng(9)
    torch = G.torch_()
    x, x64 = rows(rng, 50, 640, 640, "bf16")
    dy, dy64 = rows(rng, 50, 640, 640, "bf16")
    _, mean, rstd = HO.layer_norm(x64, eps=1e-5)
    ws = torch.empty(B.rwkvq_layer_norm_backward_workspace_size(50, 1, 640), dtype=torch.uint8, device="cuda")
    B.rwkvq_layer_norm_backward(dy, x, B.BF16, 50, 1, 640, None, f32(mean), f32(rstd), dy, None, None, ws)
    want, _, _ = HO.layer_norm_backward(dy64, x64)
    assert np.abs(host(dy, "bf16") - want).max() <= 2.0 ** -7 * np.abs(want).max()


def test_norm_gradients_against_differences():
    """<gradient, direction> against the central difference of the oracle's forward pass: the gradients are binary32 values of
    inputs that binary32 holds, so both sides agree to the rounding of 300 x 96 products (2^-24 each) and the step's h^2."""
    rng = np.random.default_rng(11)
    torch = G.torch_()
    M, groups, n = 60, 2, 48
    x, x64 = rows(rng, M, 96, 96, "f32")
    dy, dy64 = rows(rng, M, 96, 96, "f32")
    w = rng.standard_normal(96).astype(np.float32)
    y, mean, rstd = torch.empty_like(x), torch.empty((M, groups), device="cuda"), torch.empty((M, groups), device="cuda")
    B.rwkvq_layer_norm(x, B.F32, M, groups, n, f32(w), None, 1e-5, y, mean, rstd)
    dx, dw, db = torch.empty_like(x), torch.empty(96, device="cuda"), torch.empty(96, device="cuda")
    ws = torch.empty(B.rwkvq_layer_norm_backward_workspace_size(M, groups, n), dtype=torch.uint8, device="cuda")
    B.rwkvq_layer_norm_backward(dy, x, B.F32, M, groups, n, f32(w), mean, rstd, dx, dw, db, ws)
    L = lambda x, w: (HO.layer_norm(x, w, None, 1e-5, groups)[0] * dy64).sum()
    for _ in range(3):
        d, h = rng.standard_normal(x64.shape), 1e-4
        scale = np.abs(wide32(dx) * d).sum()
        assert abs((wide32(dx) * d).sum() - (L(x64 + h * d, w) - L(x64 - h * d, w)) / (2 * h)) <= 2e-6 * scale
        d = rng.standard_normal(96)
        assert abs((wide32(dw) * d).sum() - (L(x64, w + h * d) - L(x64, w - h * d)) / (2 * h)) <= 2e-6 * np.abs(wide32(dw) * d).sum()


def test_norm_rows_beyond_32_bits():
    """Rows that begin more than 2^31 elements behind the first one."""
    torch = G.torch_()
    stride, M, n = (1 << 28) + 8, 10, 320
    x = torch.empty(stride * (M - 1) + n, dtype=torch.int16, device="cuda")
    rng = np.random.default_rng(12)
    a = synth.f32_to_f16_bits(rng.standard_normal((M, n)).astype(np.float32))
    for m in range(M):
        x[m * stride:m * stride + n] = torch.from_numpy(a[m].view(np.int16)).cuda()
    B.rwkvq_layer_norm(x, B.F16, M, 1, n, None, None, 1e-5, x, x_stride=stride, y_stride=stride)
    want, mean, rstd = HO.layer_norm(widen(a, "f16"))
    got = np.stack([widen(x[m * stride:m * stride + n].cpu().numpy().view(np.uint16), "f16") for m in range(M)])
    assert np.abs(got - want).max() <= 2.0 ** -11 * 1.01 * np.abs(want).max() + 1e-5
    del x
    torch.cuda.empty_cache()


def test_norm_on_another_stream_and_in_a_graph():
    torch = G.torch_()
    rng = np.random.default_rng(13)
    M, n = 64, 1024
    x, _ = rows(rng, M, n, n, "bf16")
    dy, _ = rows(rng, M, n, n, "bf16")
    w = f32(rng.standard_normal(n))
    y, dx = torch.empty_like(x), torch.empty_like(x)
    mean, rstd, dw, db = (torch.empty(s, device="cuda") for s in (M, M, n, n))
    ws = torch.empty(B.rwkvq_layer_norm_backward_workspace_size(M, 1, n), dtype=torch.uint8, device="cuda")

    def both():
        B.rwkvq_layer_norm(x, B.BF16, M, 1, n, w, None, 1e-5, y, mean, rstd)
        B.rwkvq_layer_norm_backward(dy, x, B.BF16, M, 1, n, w, mean, rstd, dx, dw, db, ws)

    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        both()
    s.synchronize()
    outs = [y, mean, rstd, dx, dw, db]
    first = [t.clone() for t in outs]
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        both()
    for _ in range(3):
        x.copy_(x.roll(1, 0)); dy.copy_(dy.roll(1, 0))
        for t in outs:
            t.zero_()
        g.replay()
        torch.cuda.synchronize()
        replayed = [t.clone() for t in outs]
        both()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(replayed, outs))
    assert torch.equal(first[0].roll(3, 0), y)             # rows do not depend on their place
