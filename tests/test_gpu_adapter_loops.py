"""GPU parity of the adapters where the kernels' loops go round several times, as they do in large calls: several shares of the columns in a slice, several
slices of a tile of 32 rows, pieces of up to 4096 tokens in the sums over tokens.  What each case has is checked on the host (test_adapter_plan.py).

Bars: those of test_gpu_adapters.py, which count the roundings of any size."""
import copy

import numpy as np
import pytest

from paper_2505_03803_amd import binding as B

import adapter_cases as C
import fast_masks
import gpu_util as G
from test_gpu_adapters import Case, backward, check_backward, check_forward, forward

pytestmark = pytest.mark.gpu
torch = G.torch_()


class Large(Case):
    """The oracle's masks in arrays, made once."""

    def stays(self, i):
        if not self.p:
            return 1.0
        if not hasattr(self, "masks"):
            self.masks = {}
        if i not in self.masks:
            stays, factor = fast_masks.keep(self.seed, self.p, self.all, self.K, call=i)
            self.masks[i] = stays * factor
        return self.masks[i]


@pytest.mark.parametrize("case", [c for c, *_ in C.SUMS], ids=lambda c: "x".join(map(str, c[2:])))
@pytest.mark.parametrize("dt,p", [("f16", 0.0), ("bf16", 0.3), ("f16", 0.3), ("bf16", 0.0)])
def test_sums_over_many_tokens(case, dt, p):
    lens, ids, n, r, K, N, mats = case
    c = Large(lens, ids, n, r, K, N, dt, mats=mats, p=p, tail=3)
    print(case, dt, p, flush=True)
    hs = forward(c, dt)[1]
    check_backward(c, hs, *backward(c, hs))


@pytest.mark.parametrize("case", [c for c, *_ in C.ROUNDS], ids=lambda c: "%dx%s" % (c[3], sum(c[0])))
@pytest.mark.parametrize("dt,y_dt,p", [("f16", "f16", 0.0), ("bf16", "bf16", 0.3), ("f16", "f32", 0.3), ("bf16", "f32", 0.0), ("f16", "f16", 0.3), ("bf16", "bf16", 0.0)])
def test_columns_in_several_rounds(case, dt, y_dt, p):
    lens, ids, n, r = case
    c = Large(lens, ids, n, r, C.NARROW, C.WIDE, dt, mats=8, p=p, tail=3)
    print(case, dt, y_dt, p, flush=True)
    check_forward(c, y_dt, *forward(c, y_dt))


@pytest.mark.parametrize("case", [c for c, *_ in C.ROUNDS], ids=lambda c: "%dx%s" % (c[3], sum(c[0])))
@pytest.mark.parametrize("dt,p", [("f16", 0.0), ("bf16", 0.3), ("f16", 0.3), ("bf16", 0.0)])
def test_gradients_of_columns_in_several_rounds(case, dt, p):
    lens, ids, n, r = case
    c = Large(lens, ids, n, r, C.WIDE, C.NARROW, dt, mats=8, p=p, tail=3)
    print(case, dt, p, flush=True)
    hs = forward(c, dt)[1]
    check_backward(c, hs, *backward(c, hs))


@pytest.mark.parametrize("case", [c for c, *_ in C.GATHERED], ids=lambda c: "x".join(map(str, c)))
@pytest.mark.parametrize("dt,y_dt", [("f16", "f16"), ("bf16", "bf16"), ("f16", "f32")])
def test_single_tokens_in_several_rounds(case, dt, y_dt):
    tokens, n, r = case
    ids = np.random.default_rng(tokens).integers(-1, n, size=tokens).tolist()
    c = Large([1] * tokens, ids, n, r, C.NARROW, C.WIDE, dt, mats=8, ragged=False)
    check_forward(c, y_dt, *forward(c, y_dt))
    if y_dt == dt:
        c = Large([1] * tokens, ids, n, r, C.WIDE, C.NARROW, dt, mats=8, ragged=False)
        hs = forward(c, dt)[1]
        check_backward(c, hs, *backward(c, hs))


@pytest.mark.parametrize("case", [c for c, *_ in C.SLICES], ids=lambda c: "x".join(map(str, c[2:])))
@pytest.mark.parametrize("dt,y_dt", [("f16", "f16"), ("bf16", "bf16"), ("bf16", "f32")])
def test_slices_of_tiles_of_32_rows(case, dt, y_dt):
    """Columns next to the ends of slices and rounds, and a sample of the others; h of every row."""
    lens, ids, n, r, K, N, mats = case
    c = Large(lens, ids, n, r, K, N, dt, mats=mats, tail=3)
    ys, hs, bases = forward(c, y_dt)
    rng = np.random.default_rng(N)
    cols = np.unique(np.concatenate([rng.integers(0, N, size=300), np.arange(0, N, 64), np.arange(63, N, 64), [N - 1]]))
    at = torch.from_numpy(np.concatenate([cols, np.arange(N, N + c.pad)])).cuda()
    some = copy.copy(c)
    some.N, some.b = len(cols), [b[:, torch.from_numpy(cols).cuda()] for b in c.b]
    check_forward(some, y_dt, [y[:, at] for y in ys], hs, [b[:, at] for b in bases])


@pytest.mark.parametrize("shape", [([20, 30, 10], [0, 1, 0], 2, 16, 72, 40), ([700, 613], [1, 0], 2, 32, 72, 40)], ids=lambda s: str(sum(s[0])))
def test_offsets_out_of_order_leave_other_rows(shape):
    """Rows in front of the first and behind the last one of y, h, dx and the padding beside them are not touched, whatever the offsets hold."""
    c = Case(*shape, "bf16", mats=8, tail=4)
    M, guard, stride_y, stride_x = c.all, 96, c.N + 8, c.K + 8
    whole = lambda stride, t: [torch.full((M + 2 * guard, stride), 9.0, dtype=t, device="cuda") for _ in range(8)]  # noqa: E731
    inner = lambda ts: [t[guard:guard + M] for t in ts]  # noqa: E731
    last = M - 4
    for offsets in ([0, 20, 50, 2000], [-5, 20, 10, 64], [2 ** 30] * 4, [-2 ** 31, 20, 2 ** 31 - 1, 0], [last, 0, last, -1], [M, M, 3, M]):
        c.offsets.copy_(torch.tensor(offsets[:len(c.lens) + 1], dtype=torch.int32))
        y, h, dx = whole(stride_y, torch.bfloat16), whole(c.r, torch.float32), whole(stride_x, torch.bfloat16)
        B.rwkvq_adapters(c.rows, B.AdapterTable(c.a, c.b, c.x, inner(y), hs=inner(h), x_strides=stride_x, y_strides=stride_y), B.BF16, B.BF16)
        das, dbs = [[torch.full(t.shape, 9.0, device="cuda") for t in ts] for ts in (c.a, c.b)]
        table = B.AdapterGradTable(c.a, c.b, c.x, inner(h), c.dy, inner(dx), das, dbs, x_strides=stride_x, dy_strides=c.N + c.pad, dx_strides=stride_x)
        n = B.rwkvq_adapters_backward_workspace_size(c.rows, table)
        ws = torch.full((n + 64,), 0x5A, dtype=torch.uint8, device="cuda")
        B.rwkvq_adapters_backward(c.rows, table, B.BF16, ws)
        assert bool((ws[n:] == 0x5A).all())
        for t, width in [(t, c.N) for t in y] + [(t, c.r) for t in h] + [(t, c.K) for t in dx]:
            assert bool((t[:guard] == 9.0).all()) and bool((t[guard + M:] == 9.0).all()) and bool((t[:, width:] == 9.0).all()), offsets
