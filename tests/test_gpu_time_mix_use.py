"""The time-mixing block as programs hold it: a captured graph without the block's name."""
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
