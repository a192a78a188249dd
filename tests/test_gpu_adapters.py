"""GPU parity of low-rank adapters and their gradients with the binary64 oracle.

Bars.  Matrix cores add 32 products and the running sum, counted as 32 roundings of 2^-23 (nearest or not).  h: a wavefront takes 64 of every 512 of
the K columns, 64 ceil(K / 512) roundings, then four sums and a factor: gamma(K) = (64 ceil(K / 512) + 8) 2^-23 of sum |A| |x|.  y: h in parts, off by
2^-16 of itself (bf16) or 2^-22 of the row's largest (fp16), 2^-24 where y is binary32 (2^-23 with the scale's rounding), at most 32 ceil(3 rank / 32) + 4
further roundings, and half a step of y's type.  Gradients of A and B: a piece of up to 4096 tokens adds at most five products for every 32 tokens, 160
roundings, and every piece, of 64 rows at least, one more; operands of 24 bits, 2^-22 with the products left out."""
import numpy as np
import pytest

from oracle import tuning_oracle as TO
from paper_2505_03803_amd import binding as B

import gpu_util as G
from test_gpu_dropout import TYPES, half_step, seed_of

pytestmark = pytest.mark.gpu
torch = G.torch_()


def gamma(K):
    return (64 * -(-K // 512) + 8) * 2.0 ** -23


def f64(t):
    return t.cpu().double().numpy()


class Case:
    """Inputs of a call, on the GPU and in binary64.  tail: rows of no sequence behind the last one."""

    def __init__(self, lens, ids, n, r, K, N, dt, mats=1, p=0.0, ragged=True, tail=0, pad=8, seed=0):
        torch.manual_seed(seed + sum(lens) + K + N + r)
        self.lens, self.ids, self.n, self.r, self.K, self.N, self.dt, self.mats, self.p = lens, ids, n, r, K, N, dt, mats, p
        self.t, self.M, self.all, self.pad = TYPES[dt], sum(lens), sum(lens) + tail, pad
        i32 = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")  # noqa: E731
        self.seed = (2 ** 60 + 7, 2 ** 33 - 2)
        self.scales = torch.rand(n) * 1.5 + 0.5
        self.offsets = i32(np.concatenate([[0], np.cumsum(lens)]))
        self.rows = B.AdapterRows(len(lens), self.all, n, r, offsets=self.offsets if ragged else None, adapters=i32(ids), scales=self.scales.cuda(),
                                  seed=seed_of(*self.seed) if p else None, p=p)
        rand = lambda *shape: torch.randn(*shape).to(self.t).cuda()  # noqa: E731
        self.a = [(torch.randn(n, r, K) * K ** -0.5).to(self.t).cuda() for _ in range(mats)]
        self.b = [(torch.randn(n, N, r) * 0.2).to(self.t).cuda() for _ in range(mats)]
        self.x = [rand(self.all, K + pad) for _ in range(mats)]
        self.dy = [rand(self.all, N + pad) for _ in range(mats)]

    def stays(self, i):
        if not self.p:
            return 1.0
        stays, factor = TO.keep(self.seed, self.p, self.all, self.K, call=i)
        return stays * factor

    def dropped(self, i):
        x = f64(self.x[i])[:, :self.K]
        return np.where(self.stays(i) == 0.0, 0.0, x * self.stays(i)) if self.p else x


def forward(c, y_dt, base=True, h=True, in_place=False):
    yt, pad = TYPES[y_dt], c.pad
    bases = [torch.randn(c.all, c.N + pad).to(yt).cuda() for _ in range(c.mats)] if base else None
    ys = [b.clone() for b in bases] if in_place else [torch.full((c.all, c.N + pad), 9.0, dtype=yt, device="cuda") for _ in range(c.mats)]
    hs = [torch.full((c.all, c.r), 9.0, device="cuda") for _ in range(c.mats)] if h else None
    table = B.AdapterTable(c.a, c.b, c.x, ys, bases=ys if in_place else bases, hs=hs, x_strides=c.K + pad, base_strides=c.N + pad if base else 0,
                           y_strides=c.N + pad)
    B.rwkvq_adapters(c.rows, table, B.DTYPES[c.dt], B.DTYPES[y_dt])
    return ys, hs, bases


def has_adapter(c):
    live = np.zeros(c.all, dtype=bool)
    for _, f, e in TO.adapter_rows(c.lens, c.ids, c.n):
        live[f:e] = True
    return live


def check(got, want, bar, what):
    bad = ~(np.abs(got - want) <= bar)
    assert not bad.any(), (what, int(bad.sum()), float(np.nanmax(np.abs(got - want) / np.maximum(bar, 1e-300))), np.argwhere(bad)[:4])


def check_forward(c, y_dt, ys, hs, bases):
    live, yt = has_adapter(c), TYPES[y_dt]
    for i in range(c.mats):
        x, a, b, s = c.dropped(i)[:c.M], f64(c.a[i]), f64(c.b[i]), c.scales.double().numpy()
        base = f64(bases[i])[:c.M, :c.N] if bases else np.zeros((c.M, c.N))
        y, h = TO.adapters(x, a, b, c.lens, c.ids, s, base)
        dh, dy = np.zeros_like(h), np.zeros_like(y)
        for id_, f, e in TO.adapter_rows(c.lens, c.ids, c.n):
            dh[f:e] = gamma(c.K) * (np.abs(x[f:e]) @ np.abs(a[id_]).T)
            size = np.abs(h[f:e])
            part = (size * (2.0 ** -16 if c.dt == "bf16" else 0.0) + (size.max(1, keepdims=True) * 2.0 ** -22 if c.dt == "f16" else 0.0)
                    if y_dt != "f32" else 2.0 ** -22 * size)
            more = (32 * -(-3 * c.r // 32) + 4) * 2.0 ** -23
            dy[f:e] = s[id_] * ((dh[f:e] + part + more * size) @ np.abs(b[id_]).T) + 2.0 ** -23 * np.abs(base[f:e])
        got = f64(ys[i])
        step = half_step(yt, torch.from_numpy(np.abs(y) + dy)).numpy()
        check(got[:c.M, :c.N], y, dy + step, "y")
        assert (got[c.M:] == 9.0).all() and (got[:, c.N:] == (f64(bases[i])[:, c.N:] if (got[0, c.N:] != 9.0).any() else 9.0)).all()
        if bases:
            rest = torch.from_numpy(~live[:c.M]).cuda()
            assert torch.equal(ys[i][:c.M, :c.N][rest], bases[i][:c.M, :c.N][rest])
        if hs:
            check(f64(hs[i])[:c.M], h, dh, "h")
            assert (f64(hs[i])[c.M:] == 9.0).all()


# lengths from none to many, one of them a piece of tiles; adapters shared, missing, outside; widths below a step, odd multiples of 8
SHAPES = [
    ([1], [0], 1, 8, 8, 8), ([1], [2], 3, 16, 4096, 1000), ([1] * 20, list(range(5)) * 4, 5, 16, 520, 264), ([16], [0], 1, 16, 512, 64),
    ([17], [0], 1, 24, 72, 136), ([3, 0, 40, 1, 33], [1, 0, 0, -1, 1], 2, 32, 264, 200), ([5, 64, 2], [7, 0, -5], 3, 48, 1000, 328),
    ([100], [1], 2, 64, 1032, 520), ([31, 32, 33], [0, 0, 1], 2, 128, 584, 72), ([200, 7], [0, 1], 2, 120, 40, 2056),
    ([0, 0, 9, 0], [0, 1, 1, 0], 2, 8, 4104, 16),
    ([2, 2, 2, 2], [0, -1, 1, 0], 2, 40, 64, 64),
]


@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s[2:])))
@pytest.mark.parametrize("dt,y_dt", [("f16", "f16"), ("bf16", "bf16"), ("f16", "f32"), ("bf16", "f32"), ("f16", "bf16"), ("bf16", "f16")])
def test_forward(shape, dt, y_dt):
    c = Case(*shape, dt, tail=3)
    print(shape, dt, y_dt, flush=True)
    check_forward(c, y_dt, *forward(c, y_dt))


@pytest.mark.parametrize("dt", ["f16", "bf16"])
@pytest.mark.parametrize("mats", [1, 4, 8, 9])
def test_forward_of_several_matrices_with_dropout(dt, mats):
    c = Case([20, 3, 1], [1, 0, 1], 2, 16, 104, 72, dt, mats=mats, p=0.25)
    check_forward(c, dt, *forward(c, dt))


@pytest.mark.parametrize("lens,ids", [([1] * 33, [0, 1, -1] * 11), ([12] * 5, [0, 1, 1, 0, 3]), ([40] * 3, [1, 1, 0])])
def test_forward_of_equal_lengths(lens, ids):
    for base, h, in_place in ((True, True, False), (False, False, False), (True, False, True)):
        c = Case(lens, ids, 2, 16, 136, 88, "bf16", ragged=False)
        ys, hs, bases = forward(c, "bf16", base=base, h=h, in_place=in_place)
        check_forward(c, "bf16", ys, hs, bases)


def backward(c, hs, base=True, dx=True):
    pad, like = c.pad, lambda *shape: torch.full(shape, 9.0, device="cuda")
    bases = [torch.randn(c.all, c.K + pad).to(c.t).cuda() for _ in range(c.mats)] if base else None
    dxs = [torch.full((c.all, c.K + pad), 9.0, dtype=c.t, device="cuda") for _ in range(c.mats)] if dx else None
    das, dbs = [like(c.n, c.r, c.K) for _ in range(c.mats)], [like(c.n, c.N, c.r) for _ in range(c.mats)]
    table = B.AdapterGradTable(c.a, c.b, c.x, hs, c.dy, dxs, das, dbs, bases=bases, x_strides=c.K + pad, dy_strides=c.N + pad,
                               base_strides=c.K + pad if base else 0, dx_strides=c.K + pad)
    n = B.rwkvq_adapters_backward_workspace_size(c.rows, table)
    ws = torch.full((n + 64,), 0x5A, dtype=torch.uint8, device="cuda")
    B.rwkvq_adapters_backward(c.rows, table, B.DTYPES[c.dt], ws)
    assert bool((ws[n:] == 0x5A).all())
    return dxs, das, dbs, bases


def check_backward(c, hs, dxs, das, dbs, bases):
    live = has_adapter(c)
    for i in range(c.mats):
        x, dy, h = c.dropped(i)[:c.M], f64(c.dy[i])[:c.M, :c.N], f64(hs[i])[:c.M]
        a, b, s = f64(c.a[i]), f64(c.b[i]), c.scales.double().numpy()
        stays = c.stays(i)[:c.M] if c.p else 1.0
        dx, da, db = TO.adapters_backward(x, dy, h, a, b, c.lens, c.ids, s, stays)
        base = f64(bases[i])[:c.M, :c.K] if bases else np.zeros_like(dx)
        ddx, dda, ddb, pieces = np.zeros_like(dx), np.zeros_like(da), np.zeros_like(db), np.zeros(c.n)
        for id_, f, e in TO.adapter_rows(c.lens, c.ids, c.n):
            g, size = s[id_] * (dy[f:e] @ b[id_]), s[id_] * (np.abs(dy[f:e]) @ np.abs(b[id_]))
            dg = gamma(c.N) * size
            part = np.abs(g) * 2.0 ** -16 if c.dt == "bf16" else np.abs(g).max(1, keepdims=True) * 2.0 ** -22
            more = (32 * -(-3 * c.r // 32) + 4) * 2.0 ** -23
            ddx[f:e] = (dg + part + more * np.abs(g)) @ np.abs(a[id_])
            pieces[id_] += (e - f) // 64 + 2
            depth = (160 * -(-min(e - f, 4096) // 32)) * 2.0 ** -23 + 2.0 ** -22
            dda[id_] += (dg + depth * np.abs(g)).T @ np.abs(x[f:e])
            ddb[id_] += s[id_] * (np.abs(dy[f:e]).T @ (depth * np.abs(h[f:e])))
            dda[id_] += (pieces[id_] + 2) * 2.0 ** -23 * (np.abs(g).T @ np.abs(x[f:e]))
            ddb[id_] += (pieces[id_] + 2) * 2.0 ** -23 * s[id_] * (np.abs(dy[f:e]).T @ np.abs(h[f:e]))
        check(f64(das[i]), da, dda, "da")
        check(f64(dbs[i]), db, ddb, "db")
        if dxs:
            got, want = f64(dxs[i]), dx + base
            bar = ddx * stays + 2.0 ** -23 * np.abs(base)
            check(got[:c.M, :c.K], want, bar + half_step(c.t, torch.from_numpy(np.abs(want) + bar)).numpy(), "dx")
            assert (got[c.M:] == 9.0).all() and (got[:, c.K:] == 9.0).all()
            if bases:
                rest = torch.from_numpy(~live[:c.M]).cuda()
                assert torch.equal(dxs[i][:c.M, :c.K][rest], bases[i][:c.M, :c.K][rest])


@pytest.mark.parametrize("shape", SHAPES + [([700], [0], 1, 16, 200, 136), ([300, 290], [1, 1], 2, 64, 136, 264)], ids=lambda s: "x".join(map(str, s[2:])))
@pytest.mark.parametrize("dt", ["f16", "bf16"])
def test_backward(shape, dt):
    c = Case(*shape, dt, tail=3)
    print(shape, dt, flush=True)
    hs = forward(c, dt)[1]
    check_backward(c, hs, *backward(c, hs))


@pytest.mark.parametrize("dt", ["f16", "bf16"])
@pytest.mark.parametrize("base,dx", [(True, True), (False, True), (False, False)])
def test_backward_with_dropout(dt, base, dx):
    c = Case([50, 0, 33, 2], [1, 0, 1, -1], 3, 24, 264, 72, dt, mats=3, p=0.3)
    hs = forward(c, dt)[1]
    check_backward(c, hs, *backward(c, hs, base=base, dx=dx))


def test_more_than_eight_matrices_backward():
    c = Case([40, 9], [1, 0], 2, 16, 72, 136, "bf16", mats=10, p=0.1)
    hs = forward(c, "bf16")[1]
    check_backward(c, hs, *backward(c, hs))


# tiles of 32 rows: eight matrices, whose tiles of 16 together have more than 20000 values of the rank
MANY = [([300, 0, 340, 33, 31, 200], [0, 1, 1, 0, -1, 1], 2, 64, 136, 72), ([500, 40, 401], [1, -1, 0], 2, 48, 72, 264),
        ([1000, 40, 700], [1, 5, 0], 2, 24, 72, 200), ([1300], [0], 1, 32, 104, 40)]


@pytest.mark.parametrize("shape", MANY, ids=lambda s: "x".join(map(str, s[2:])))
@pytest.mark.parametrize("dt,y_dt,p", [("f16", "f16", 0.0), ("bf16", "bf16", 0.3), ("f16", "f32", 0.3), ("bf16", "f32", 0.0), ("bf16", "f16", 0.0)])
def test_many_rows(shape, dt, y_dt, p):
    c = Case(*shape, dt, mats=8, p=p, tail=5)
    print(shape, dt, y_dt, p, flush=True)
    check_forward(c, y_dt, *forward(c, y_dt))


@pytest.mark.parametrize("shape", MANY, ids=lambda s: "x".join(map(str, s[2:])))
@pytest.mark.parametrize("dt,p", [("f16", 0.0), ("bf16", 0.0), ("bf16", 0.3), ("f16", 0.3)])
def test_many_rows_backward(shape, dt, p):
    c = Case(*shape, dt, mats=8, p=p, tail=5)
    print(shape, dt, p, flush=True)
    hs = forward(c, dt)[1]
    check_backward(c, hs, *backward(c, hs))


@pytest.mark.parametrize("rank", [8, 24, 32, 40, 64, 120])
@pytest.mark.parametrize("dt,y_dt", [("f16", "f16"), ("bf16", "bf16"), ("bf16", "f32")])
def test_a_row_alone(rank, dt, y_dt):
    """The bits of a row do not depend on the rows beside it: in tiles of 32 and of 16 rows, gathered from single tokens, in slices of the columns, alone."""
    mats, M, K, N = 8, 2000, 1160, 328
    big = Case([M], [1], 2, rank, K, N, dt, mats=mats)
    want, hs, bases = forward(big, y_dt)
    table = lambda c, rows, ys, at: B.AdapterTable(  # noqa: E731
        c.a, c.b, [x[at:at + rows] for x in c.x], ys, bases=[b[at:at + rows] for b in bases], x_strides=K + 8, base_strides=N + 8, y_strides=N + 8)
    ids = lambda n: torch.ones(n, dtype=torch.int32, device="cuda")  # noqa: E731
    for seqs, rows, at in ((1, 1, 777), (1, 15, 32), (1, 45, 100), (40, 40, 64), (20, 40, 1000), (3, 300, 1700)):
        ys = [torch.full((rows, N + 8), 9.0, dtype=TYPES[y_dt], device="cuda") for _ in range(mats)]
        few = B.AdapterRows(seqs, rows, 2, rank, adapters=ids(seqs), scales=big.scales.cuda())
        B.rwkvq_adapters(few, table(big, rows, ys, at), B.DTYPES[dt], B.DTYPES[y_dt])
        for y, w in zip(ys, want):
            assert torch.equal(y[:, :N], w[at:at + rows, :N]), (seqs, rows, at)


@pytest.mark.parametrize("n,ids", [(300, lambda i: 0), (2048, lambda i: i * 7 % 5 - 1), (2048, lambda i: 1 if i > 2040 else 0), (2049, lambda i: i % 3),
                                   (64, lambda i: -1)])
@pytest.mark.parametrize("rank", [8, 40, 120])
def test_single_tokens_of_many_users(n, ids, rank):
    c = Case([1] * n, [ids(i) for i in range(n)], 4, rank, 72, 136, "bf16", ragged=False)
    check_forward(c, "bf16", *forward(c, "bf16"))


@pytest.mark.parametrize("n,adapters", [(2, 5), (16, 2), (17, 2), (90, 3), (200, 300)])
@pytest.mark.parametrize("rank,dt", [(8, "f16"), (40, "bf16"), (128, "bf16")])
def test_single_tokens_backward(n, adapters, rank, dt):
    rng = np.random.default_rng(n)
    c = Case([1] * n, rng.integers(-1, adapters, size=n).tolist(), adapters, rank, 136, 72, dt, mats=2, ragged=False)
    hs = forward(c, dt)[1]
    check_backward(c, hs, *backward(c, hs))


@pytest.mark.parametrize("ragged", [False, True])
def test_one_adapter_for_all(ragged):
    """No numbers of adapters: all sequences have the first, also where gradients are summed over them."""
    c = Case([20, 20, 20, 20], [0] * 4, 1, 24, 72, 136, "bf16", mats=2, p=0.2, tail=0)
    c.rows = B.AdapterRows(4, 80, 1, 24, offsets=c.offsets if ragged else None, scales=c.scales.cuda(), seed=c.rows.keep[3], p=c.p)
    ys, hs, bases = forward(c, "bf16")
    check_forward(c, "bf16", ys, hs, bases)
    check_backward(c, hs, *backward(c, hs))


def test_sixty_four_matrices():
    c = Case([9, 1], [1, 0], 2, 8, 40, 24, "f16", mats=64, p=0.1)
    ys, hs, bases = forward(c, "f16")
    check_forward(c, "f16", ys, hs, bases)
    check_backward(c, hs, *backward(c, hs))


def test_offsets_stay_in_bounds():
    """Offsets that descend or pass the last row are limited to the rows that there are; those in order have their results."""
    c = Case([20, 30, 10], [0, 1, 0], 2, 16, 72, 40, "bf16", tail=4)
    good = forward(c, "bf16", base=False)[0][0].clone()
    for offsets in ([0, 20, 50, 2000], [-5, 20, 10, 64], [2 ** 30] * 4, [-2 ** 31, 20, 2 ** 31 - 1, 0]):
        c.offsets.copy_(torch.tensor(offsets, dtype=torch.int32))
        ys, hs, _ = forward(c, "bf16", base=False)
        if offsets[1] == 20:
            assert torch.equal(ys[0][:20], good[:20])
        dxs = backward(c, hs)[0]
        assert bool((ys[0][:, c.N:] == 9.0).all()) and bool((dxs[0][:, c.K:] == 9.0).all())


def test_two_streams():
    """Calls that run side by side, each with a workspace of its own."""
    cases = [Case([700, 41], [0, 1], 2, 64, 264, 520, "bf16", mats=2, p=0.1, seed=i) for i in range(2)]
    want = []
    for c in cases:
        hs = forward(c, "bf16", base=False)[1]
        want.append((hs, backward(c, hs, base=False)[:3]))
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in range(2)], [None, None]
    for _ in range(3):
        for i, c in enumerate(cases):
            with torch.cuda.stream(streams[i]):
                hs = forward(c, "bf16", base=False)[1]
                got[i] = (hs, backward(c, hs, base=False)[:3])
    torch.cuda.synchronize()
    for w, g in zip(want, got):
        assert all(torch.equal(a, b) for a, b in zip(w[0], g[0]))
        for a, b in zip(w[1], g[1]):
            assert all(torch.equal(x, y) for x, y in zip(a, b))


def test_rows_far_apart():
    """Places beyond 2^32 elements: rows 2^27 apart."""
    far, M = 1 << 27, 40
    c = Case([M - 3, 3], [0, 1], 2, 16, 64, 40, "bf16", pad=8)
    x, y = (torch.empty(M * far - far + 64, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    rows = lambda t, n: t.as_strided((M, n), (far, 1))  # noqa: E731
    rows(x, 64).copy_(c.x[0][:, :64])
    h, plain = torch.empty(M, 16, device="cuda"), torch.empty(M, 40, dtype=torch.bfloat16, device="cuda")
    B.rwkvq_adapters(c.rows, B.AdapterTable(c.a, c.b, [x], [y], hs=[h], x_strides=far, y_strides=far), B.BF16, B.BF16)
    B.rwkvq_adapters(c.rows, B.AdapterTable(c.a, c.b, c.x, [plain], x_strides=72), B.BF16, B.BF16)
    assert torch.equal(rows(y, 40), plain)
    # gradients: dy in y's place, dx in another
    dx = torch.empty_like(x)
    for strided in (True, False):
        da, db = torch.empty(2, 16, 64, device="cuda"), torch.empty(2, 40, 16, device="cuda")
        near = torch.empty(M, 64, dtype=torch.bfloat16, device="cuda")
        if strided:
            table = B.AdapterGradTable(c.a, c.b, [x], [h], [y], [dx], [da], [db], x_strides=far, dy_strides=far, dx_strides=far)
        else:
            table = B.AdapterGradTable(c.a, c.b, c.x, [h], [plain], [near], [da], [db], x_strides=72)
        ws = torch.empty(B.rwkvq_adapters_backward_workspace_size(c.rows, table), dtype=torch.uint8, device="cuda")
        B.rwkvq_adapters_backward(c.rows, table, B.BF16, ws)
        if strided:
            first = da.clone(), db.clone()
    assert torch.equal(first[0], da) and torch.equal(first[1], db) and torch.equal(rows(dx, 64), near)


def test_gradients_are_differences():
    """Losses of the kernels' own binary32 outputs: y is linear in A and in B, so a difference of steps that 16-bit types hold is the gradient up to
    the bars of two outputs."""
    c = Case([30, 20], [0, 1], 2, 8, 64, 40, "bf16", p=0.2)
    hs = forward(c, "f32")[1]
    dxs, das, dbs, _ = backward(c, hs, base=False)
    dy = c.dy[0][:, :c.N].double()
    rng = np.random.default_rng(0)
    for which, grad in ((c.a, das[0]), (c.b, dbs[0]), (c.x, dxs[0])):
        for _ in range(5):
            flat = which[0].view(-1)
            at = int(rng.integers(flat.numel()))
            if which is c.x and at % (c.K + c.pad) >= c.K:
                continue
            keep, out = flat[at].clone(), []
            for step in (4.0, -4.0):
                flat[at] = step
                ys = forward(c, "f32", base=False)[0]
                out.append((ys[0][:, :c.N].double() * dy).sum())
            flat[at] = keep
            slope, want = float(out[0] - out[1]) / 8.0, float(grad.reshape(-1)[at] if which is not c.x else dxs[0].view(-1)[at])
            # two losses of 50 x 40 products of values to 30 at 2^-16 each in the worst case, over a step of 8; dx has 8 bits
            assert abs(slope - want) <= 2000 * 30 * 2.0 ** -21 / 8.0 + 2.0 ** -8 * abs(want), (slope, want)


def test_the_same_bits_and_rows_for_themselves():
    """A row's outputs do not depend on what other sequences hold, on their number or on the call."""
    c = Case([40, 9, 33], [0, 1, 0], 2, 16, 520, 264, "f16", tail=2)
    ys, hs, bases = forward(c, "f16", in_place=True)
    again = [b.clone() for b in bases]
    B.rwkvq_adapters(c.rows, B.AdapterTable(c.a, c.b, c.x, again, bases=again, x_strides=c.K + 8, base_strides=c.N + 8, y_strides=c.N + 8), B.F16, B.F16)
    assert torch.equal(again[0], ys[0])
    c.x[0][:40] = float("nan")
    c.x[0][49:60] = float("inf")
    c.x[0][82:] = float("nan")
    other, h2, _ = forward(c, "f16", base=False)
    first = f64(hs[0])
    assert np.array_equal(first[40:49], f64(h2[0])[40:49]) and np.array_equal(first[60:82], f64(h2[0])[60:82])
    assert bool(torch.isfinite(other[0][40:49, :c.N]).all()) and bool(torch.isfinite(other[0][60:82, :c.N]).all())
    assert not bool(torch.isfinite(other[0][:40, :c.N]).any()) and not bool(torch.isfinite(other[0][49:60, :c.N]).any())


@pytest.mark.parametrize("scale", [2.0 ** -12, 1.0, 2.0 ** 9])
def test_fp16_values_of_any_size(scale):
    """h far below and above fp16's range goes through its row's power of two."""
    c = Case([20], [0], 1, 16, 264, 72, "f16")
    c.x[0] = (c.x[0].float() * scale * 8).half()
    c.a[0] = (c.a[0].float() * scale).half()
    check_forward(c, "f32", *forward(c, "f32", base=False))


@pytest.mark.parametrize("dt", ["f16", "bf16"])
def test_captured_with_its_gradients(dt):
    """Both calls in a graph, replayed with other rows, adapters, lengths and seeds."""
    c = Case([20, 13, 31], [0, 1, 0], 2, 16, 136, 72, dt, p=0.2)
    like = lambda t: [torch.empty_like(v) for v in t]  # noqa: E731
    base = [torch.randn(c.all, c.N).to(c.t).cuda()]
    y, h, dx = like(base), [torch.empty(c.all, c.r, device="cuda")], [torch.empty(c.all, c.K, dtype=c.t, device="cuda")]
    da, db = [torch.empty(c.n, c.r, c.K, device="cuda")], [torch.empty(c.n, c.N, c.r, device="cuda")]

    def step(y, h, dx, da, db, ws):
        B.rwkvq_adapters(c.rows, B.AdapterTable(c.a, c.b, c.x, y, bases=base, hs=h, x_strides=c.K + 8), B.DTYPES[dt], B.DTYPES[dt])
        B.rwkvq_adapters_backward(c.rows, grads(h, dx, da, db), B.DTYPES[dt], ws)

    def grads(h, dx, da, db):
        return B.AdapterGradTable(c.a, c.b, c.x, h, c.dy, dx, da, db, x_strides=c.K + 8, dy_strides=c.N + 8)

    size = B.rwkvq_adapters_backward_workspace_size(c.rows, grads(h, dx, da, db))
    ws = torch.empty(size, dtype=torch.uint8, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(y, h, dx, da, db, ws)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(y, h, dx, da, db, ws)
    _, adapters, scales, seed = c.rows.keep
    for offsets, ids in (([0, 20, 33, 64], [0, 1, 0]), ([0, 0, 64, 64], [1, -1, 1]), ([5, 6, 40, 50], [1, 1, 0])):
        c.offsets.copy_(torch.tensor(offsets, dtype=torch.int32))
        adapters.copy_(torch.tensor(ids, dtype=torch.int32))
        seed[1] += 3
        c.x[0].normal_()
        outs = [y, h, dx, da, db]
        for t in outs:
            t[0].fill_(1.0)
        graph.replay()
        want = [[torch.ones_like(t[0])] for t in outs]
        step(*want, torch.empty_like(ws))
        torch.cuda.synchronize()
        for got, w in zip(outs, want):
            assert torch.equal(got[0], w[0])
