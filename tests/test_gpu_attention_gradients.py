"""GPU parity of linear attention's gradient of w where its terms are far apart in size, with the binary64 oracle.  Bars as in
test_gpu_attention.py: the gradient of w within (2^-15 + (tokens + 256) 2^-24) of the sum of its terms' magnitudes, whatever else a
sequence holds."""
import pytest

from test_gpu_attention import Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("w", [-1.5, -2.0])
@pytest.mark.parametrize("dt,H,D", [("bf16", 2, 64), ("f16", 2, 64), ("bf16", 2, 128), ("f16", 2, 128)])
def test_growing_heads(dt, H, D, w):
    """Short sequences of heads that grow: weights of places behind their last token are beyond binary32 and reach nothing."""
    for lens in [[1], [2], [5], [2, 5, 0, 1]] + ([[10], [40], [3, 40, 0, 7]] if dt == "bf16" else []):     # e^78 is beyond gradients in fp16
        print(f"attention w={w} lens={lens} D={D} {dt}", flush=True)
        Case(lens, H, D, dt, seed=21, w=w, scale=2.0 ** -4).check_backward()
