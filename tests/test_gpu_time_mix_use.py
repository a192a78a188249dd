"""The time-mixing block as programs hold it: a captured graph without the block's name, calls between a forward and its gradients."""
import gc
import weakref

import pytest

import gpu_util as G

pytestmark = pytest.mark.gpu


def test_a_graph_keeps_the_block_it_runs_on():
    torch = G.torch_()
    from paper_2505_03803_amd import time_mix
    block = time_mix.synthetic(256, 4, 2, 8)
    x = torch.randn(2, 256, device="cuda").half()
    plan = block.plan([1, 1], [0, 1])
    held = weakref.ref(block)
    replay = block.capture(x, plan)
    want = block.forward(x, plan).clone()                  # of empty states, which the replay starts from again
    block.state.zero_(); block.last.zero_()
    del block, plan
    gc.collect()
    assert held() is not None
    others = [torch.full((1 << 16,), 7.0, device="cuda") for _ in range(16)]
    assert torch.equal(replay(), want)
    assert all(bool((o == 7.0).all()) for o in others)


def test_gradients_only_of_what_the_block_holds():
    torch = G.torch_()
    from paper_2505_03803_amd import time_mix
    block = time_mix.synthetic(256, 4, 2, 24)
    x, y, dout = (torch.randn(20, 256, device="cuda").half() for _ in range(3))
    whole, parts, slots = block.plan([20]), block.plan([7, 13]), block.plan([1], [0])
    replay = block.capture(x[:1].contiguous(), slots)
    block.forward(x, whole)
    want = block.backward(x, dout, whole)
    again = block.backward(x[:20], dout, whole)
    assert torch.equal(want["x"], again["x"]) and torch.equal(want["w"], again["w"])
    with pytest.raises(ValueError):
        block.backward(x, dout, parts)
    with pytest.raises(ValueError):
        block.backward(y, dout, whole)
    for other in (lambda: block.forward(y, whole), lambda: block.forward(x, parts), replay):
        block.forward(x, whole)
        other()
        with pytest.raises(ValueError):
            block.backward(x, dout, whole)
    block.forward(x[:1], slots)
    with pytest.raises(ValueError):
        block.backward(x[:1], dout[:1], slots)
    block.forward(x, whole)
    assert torch.equal(block.backward(x, dout, whole)["x"], want["x"])
