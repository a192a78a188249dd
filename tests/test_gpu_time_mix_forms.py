"""The time-mixing block in bf16 and with heads other than 64 channels, against the block in binary64 as in test_gpu_time_mix.py.  The bars are
the counts of roundings given there, of 2^-8 each in bf16."""
import numpy as np
import pytest

from test_gpu_time_mix import close, params_of, plain

import gpu_util as G

pytestmark = pytest.mark.gpu
ROUNDING = {"f16": 2.0 ** -11, "bf16": 2.0 ** -8}


@pytest.mark.parametrize("lens", [[1], [70], [3, 0, 1, 20], [300]])
@pytest.mark.parametrize("dt,H", [("bf16", 4), ("bf16", 2), ("f16", 2), ("f16", 8), ("bf16", 8)])
def test_forward_and_gradients(dt, H, lens):
    print(f"time mixing {dt} heads={H} lens={lens}", flush=True)
    torch = G.torch_()
    from paper_2505_03803_amd import binding as B, time_mix
    T = sum(lens)
    block = time_mix.synthetic(256, H, 5, T, dtype=B.DTYPES[dt])
    kind = time_mix.TYPES[block.dtype]
    dense = {p: B.dequant(m).cpu().double() for p, m in block.mats.items()}
    rng = np.random.default_rng(3)
    x, dout = (torch.from_numpy(rng.standard_normal((T, 256))).to(kind) for _ in range(2))
    params, xs = params_of(block), x.double().requires_grad_()
    want = plain(block, dense, xs, lens, params)
    want.backward(dout.double())
    plan, dx = block.plan(lens), x.cuda()
    got = block.forward(dx, plan).clone()
    close(got, want, 32 * ROUNDING[dt], lens)
    again = block.forward(dx, block.plan(lens, [4, 0, 3, 1][:len(lens)]))      # from empty states of a pool: the same numbers
    assert torch.equal(got, again)
    block.forward(dx, plan)
    grads = block.backward(dx, dout.cuda(), plan)
    flat = [grads["x"], *grads["ln"], *grads["heads_norm"], grads["w"], grads["u"]]
    for name, g, p in zip(["x", "ln weight", "ln bias", "heads weight", "heads bias", "w", "u"], flat, [xs] + params):
        if name == "u" and lens == [1]:                                       # a full cancellation but for eps (test_gpu_time_mix.py)
            continue
        ref = p.grad if p.grad is not None else torch.zeros_like(p)
        if float(ref.abs().max()) == 0.0:
            assert float(g.abs().max()) == 0.0, name
        else:
            close(g, ref, 64 * ROUNDING[dt], (lens, name))
