"""GPU parity of linear attention's gradient of w where its terms are far apart in size, and of calls whose sequences are many chunks or
several segments long, with the binary64 oracle.  Bars as in test_gpu_attention.py: the gradient of w within (2^-15 + (tokens + 256) 2^-24) of the
sum of its terms' magnitudes, whatever else a sequence holds."""
import numpy as np
import pytest

from test_gpu_attention import NARROW, Case, dev, widen

pytestmark = pytest.mark.gpu


def put(case, p, rows, value):
    """Rows of r, k, v or dout replaced: by zeros, or by themselves times a factor."""
    case.bits[p][rows] = NARROW[case.dt]((widen(case.bits[p][rows], case.dt) * value).astype(np.float32))
    case.x[p] = widen(case.bits[p][:, :case.wide], case.dt).reshape(case.N, case.H, case.D)
    case.d[p] = dev(case.bits[p])


@pytest.mark.parametrize("w", [-1.5, -2.0])
@pytest.mark.parametrize("dt,H,D", [("bf16", 2, 64), ("f16", 2, 64), ("bf16", 2, 128), ("f16", 2, 128)])
def test_growing_heads(dt, H, D, w):
    """Short sequences of heads that grow: weights of places behind their last token are beyond binary32 and reach nothing."""
    for lens in [[1], [2], [5], [2, 5, 0, 1]] + ([[10], [40], [3, 40, 0, 7]] if dt == "bf16" else []):     # e^78 is beyond gradients in fp16
        print(f"attention w={w} lens={lens} D={D} {dt}", flush=True)
        Case(lens, H, D, dt, seed=21, w=w, scale=2.0 ** -4).check_backward()


@pytest.mark.parametrize("dt,H,D", [("bf16", 2, 64), ("f16", 2, 64), ("bf16", 2, 128), ("f16", 1, 104)])
def test_fast_heads_over_masked_rows(dt, H, D):
    """Rows of zeros: what the state in front leaves in the one behind is all that the gradient of w has, however little it is."""
    for T, w in ((64, 0.32), (64, 1.0), (128, 0.32), (200, 0.35), (130, 0.5)):
        print(f"attention T={T} w={w} D={D} {dt}", flush=True)
        c = Case([T], H, D, dt, seed=22, w=w, offsets=False)
        for p in ("r", "k", "dout"):
            put(c, p, slice(None), 0.0)
        c.check_backward()


@pytest.mark.parametrize("dt,H,D", [("bf16", 2, 64), ("bf16", 2, 128), ("bf16", 1, 40)])
def test_outliers_that_meet_no_decay(dt, H, D):
    """The first token's r and dout and the last one's k and v have no term in the gradient of w: rounding of what they leave elsewhere has none either."""
    for T, w in ((300, 0.01), (600, 0.002), (600, 0.4), (65, 0.05)):
        print(f"attention T={T} w={w} D={D} {dt}", flush=True)
        c = Case([T], H, D, dt, seed=23, w=w, offsets=False)
        for p in ("r", "dout"):
            put(c, p, slice(0, 1), 1e4)
        for p in ("k", "v"):
            put(c, p, slice(T - 1, T), 1e4)
        c.check_backward()


# sequences that stay whole with many chunks each, that are cut into long segments, and both kinds of heads
@pytest.mark.parametrize("lens,H,D,dt", [([600] * 4, 64, 64, "bf16"), ([900] * 3, 50, 16, "f16"), ([513, 0, 640, 1, 577], 70, 40, "bf16"),
                                         ([700, 0, 1, 333], 20, 128, "f16"), ([700, 0, 1, 333], 20, 72, "bf16"),
                                         ([700, 0, 1, 333], 20, 104, "f16"), ([520] * 2, 24, 128, "bf16")])
@pytest.mark.parametrize("w", [0.001, 0.05])
def test_many_chunks(lens, H, D, dt, w):
    print(f"attention lens={lens} H={H} D={D} {dt} w={w}", flush=True)
    c = Case(lens, H, D, dt, seed=sum(lens) + H, w=w * (1 + np.arange(H) / H), offsets=len(set(lens)) > 1)
    c.check_forward()
    c.check_backward()
    first, again = c.backward(), c.backward()
    assert all(np.array_equal(first[p], again[p]) for p in first)


@pytest.mark.parametrize("lens,w", [([10], -2.0), ([40], -2.0), ([3, 40, 0, 7], -1.5), ([64], -1.3), ([66], -1.3), ([64, 1, 65], -1.2)])
@pytest.mark.parametrize("H,D", [(2, 64), (2, 128)])
def test_growing_heads_up_to_binary32(lens, w, H, D):
    """Growth by up to e^86 over a sequence, beyond a chunk of 64 tokens as well."""
    print(f"attention w={w} lens={lens} D={D}", flush=True)
    c = Case(lens, H, D, "bf16", seed=24, w=w, scale=2.0 ** -5)
    c.check_forward()
    c.check_backward()
