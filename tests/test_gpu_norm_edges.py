"""Layer norm where a workgroup stays for several rows, forward, and at the ends of what its gradients' inputs can hold.  Bars as in
test_gpu_norm.py."""
import numpy as np
import pytest

from oracle import heads_oracle as HO
from paper_2505_03803_amd import binding as B
from test_gpu_norm import FLOOR, HALF_ULP, check, f32, gamma, host, rows, wide32, xhat_error

import gpu_util as G

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("M,groups,n", [(5000, 1, 2056), (4099, 1, 1031), (3475, 80, 64), (9001, 1, 520), (9001, 3, 33), (20011, 1, 24)])
@pytest.mark.parametrize("dt", ["f16", "bf16", "f32"])
def test_workgroups_that_stay_for_rows(M, groups, n, dt, in_place):
    print(f"norm M={M} groups={groups} n={n} {dt} in place {in_place}", flush=True)
    rng = np.random.default_rng(M + n)
    torch = G.torch_()
    wide = groups * n
    stride = wide + (8 if wide % 8 == 0 else 3)
    x, x64 = rows(rng, M, wide, stride, dt, 2.0, 0.7)
    w, b = rng.standard_normal(wide).astype(np.float32), rng.standard_normal(wide).astype(np.float32)
    before = x.clone()
    y = x if in_place else torch.full_like(x, 7)
    mean, rstd = (torch.empty((M, groups), device="cuda") for _ in range(2))
    B.rwkvq_layer_norm(x, B.DTYPES[dt], M, groups, n, f32(w), f32(b), 1e-5, y, mean, rstd, x_stride=stride, y_stride=stride)
    torch.cuda.synchronize()
    want, wm, wr = HO.layer_norm(x64, w, b, 1e-5, groups)
    bar = xhat_error(x64, groups, 1e-5) * np.abs(w) + 2.0 ** -23 * (np.abs(want) + np.abs(b))
    check(host(y[:, :wide].contiguous(), dt), want, bar + HALF_ULP[dt] * 1.01 * np.abs(want) + FLOOR[dt])
    assert torch.equal(y[:, wide:], before[:, wide:]) if in_place else bool((y[:, wide:] == 7).all())
    assert np.abs(wide32(mean) - wm).max() <= 1e-5 * np.abs(x64).max() and np.abs(wide32(rstd) / wr - 1).max() <= 1e-5


# columns behind a row's end and rows behind the last one are nobody's: what they would give, 0 times an infinity, reaches nothing
@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("M,groups,n", [(3, 1, 10), (5000, 1, 40), (7, 3, 33), (70, 1, 1031), (2111, 1, 520), (33, 1, 5000)])
def test_gradients_of_equal_values_of_any_size(M, groups, n, dt):
    print(f"norm backward of equal values M={M} groups={groups} n={n} {dt}", flush=True)
    rng = np.random.default_rng(M + n)
    torch = G.torch_()
    wide = groups * n
    dy, dy64 = rows(rng, M, wide, wide, dt)
    w = rng.standard_normal(wide).astype(np.float32)
    kind = torch.float32 if dt == "f32" else torch.bfloat16
    x = torch.full((M, wide), 1.5 * 2.0 ** 124, dtype=kind, device="cuda")               # held by bf16 as it is: no deviations, xhat = 0
    mean, rstd = torch.full((M, groups), 1.5 * 2.0 ** 124, device="cuda"), torch.full((M, groups), 256.0, device="cuda")
    dx, dw, db = torch.empty_like(x), torch.empty(wide, device="cuda"), torch.empty(wide, device="cuda")
    ws = torch.empty(B.rwkvq_layer_norm_backward_workspace_size(M, groups, n), dtype=torch.uint8, device="cuda")
    B.rwkvq_layer_norm_backward(dy, x.view(torch.int16) if dt == "bf16" else x, B.DTYPES[dt], M, groups, n, f32(w), mean, rstd,
                                dx.view(torch.int16) if dt == "bf16" else dx, dw, db, ws)
    torch.cuda.synchronize()
    g = (dy64 * w).reshape(M, groups, n)
    want = 256.0 * (g - g.mean(-1, keepdims=True)).reshape(M, wide)
    bar = 256.0 * 4 * gamma(n) * (np.abs(g) + np.abs(g).mean(-1, keepdims=True)).reshape(M, wide)
    check(dx.double().cpu().numpy(), want, bar + HALF_ULP[dt] * 1.01 * np.abs(want))
    assert float(dw.abs().max()) == 0.0
    check(wide32(db), dy64.sum(0), (M + 32) * 2.0 ** -24 * np.abs(dy64).sum(0))


@pytest.mark.parametrize("M,groups,n", [(1, 1 << 24, 1), (3, 1 << 23, 2)])
def test_more_groups_than_a_launch_has_workgroups(M, groups, n):
    """2^24 groups and more, each a workgroup of 256 threads: as many as 32 bits of threads do not count."""
    print(f"norm M={M} groups={groups} n={n}", flush=True)
    torch = G.torch_()
    gen = torch.Generator(device="cuda").manual_seed(1)
    wide, eps = groups * n, 1e-5
    x, dy = (torch.randn(M, wide, generator=gen, device="cuda").half() for _ in range(2))
    w, b = (torch.randn(wide, generator=gen, device="cuda") for _ in range(2))
    y, dx = torch.empty_like(x), torch.empty_like(x)
    mean, rstd = (torch.empty(M, groups, device="cuda") for _ in range(2))
    dw, db = torch.empty(wide, device="cuda"), torch.empty(wide, device="cuda")
    bits = lambda t: t.view(torch.int16)
    B.rwkvq_layer_norm(bits(x), B.F16, M, groups, n, w, b, eps, bits(y), mean, rstd)
    ws = torch.empty(B.rwkvq_layer_norm_backward_workspace_size(M, groups, n), dtype=torch.uint8, device="cuda")
    B.rwkvq_layer_norm_backward(bits(dy), bits(x), B.F16, M, groups, n, w, mean, rstd, bits(dx), dw, db, ws)
    z = x.double().reshape(M, groups, n)
    m = z.mean(-1, keepdim=True)
    r = 1.0 / torch.sqrt(((z - m) ** 2).mean(-1, keepdim=True) + eps)
    xhat = (z - m) * r
    each = 2 * gamma(n) * (z.abs().amax(-1, keepdim=True) + (z - m).abs().amax(-1, keepdim=True)) * r      # the bar of xhat
    want = xhat.reshape(M, wide) * w.double() + b.double()
    bar = (each * w.double().abs().reshape(groups, n)).reshape(M, wide) + 2.0 ** -23 * (want.abs() + b.double().abs())
    assert bool(((y.double() - want).abs() <= bar + HALF_ULP["f16"] * 1.01 * want.abs() + FLOOR["f16"]).all())
    d = dy.double()
    g = (d * w.double()).reshape(M, groups, n)
    c2 = (g * xhat).mean(-1, keepdim=True)
    want = (r * (g - g.mean(-1, keepdim=True) - xhat * c2)).reshape(M, wide)
    big, a2 = xhat.abs() + each, (g.abs() * (xhat.abs() + each)).mean(-1, keepdim=True)
    bar = r * (4 * gamma(n) * (g.abs() + g.abs().mean(-1, keepdim=True) + big * a2) + each * a2 + big * (g.abs() * each).mean(-1, keepdim=True))
    assert bool(((dx.double() - want).abs() <= bar.reshape(M, wide) + HALF_ULP["f16"] * 1.01 * want.abs() + FLOOR["f16"]).all())
    flat = xhat.reshape(M, wide)
    err = (each.expand(M, groups, n).reshape(M, wide) * d.abs()).sum(0) + (M + 32) * 2.0 ** -24 * (d * flat).abs().sum(0) + 2.0 ** -126
    assert bool(((dw.double() - (d * flat).sum(0)).abs() <= err).all())
    assert bool(((db.double() - d.sum(0)).abs() <= (M + 32) * 2.0 ** -24 * d.abs().sum(0) + 2.0 ** -126).all())
