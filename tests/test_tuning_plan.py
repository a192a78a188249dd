"""CPU-side checks of plans with adapters: those that a block does not have are refused."""
import types

import pytest
import torch

from paper_2505_03803_amd import binding as B
from paper_2505_03803_amd.time_mix import Adapters, TimeMix
from paper_2505_03803_amd.tuning import Tuning


def block(n):
    b = object.__new__(TimeMix)                            # what plan() looks at, without a GPU
    b.H, b.D, b.max_tokens, b.n_slots, b.device = 2, 64, 40, 5, "cpu"
    if n:
        b.adapters = types.SimpleNamespace(n=n, rank=8, p=0.1, scales=None, seeds=[None, None])
    return b


@pytest.mark.parametrize("n,lens,ids", [(0, [3], [0]), (2, [3, 4], [0]), (2, [3, 4], [0, 2]), (2, [3, 4], [-2, 0]), (2, [3], [0, 1]), (2, [3], [2 ** 31])])
def test_adapters_that_are_refused(n, lens, ids):
    with pytest.raises(ValueError):
        block(n).plan(lens, adapters=ids)


@pytest.mark.parametrize("lens,ids", [([3, 4], [1, -1]), ([1, 1], [0, 0]), ([40], [1]), ([3, 0, 5], [0, 1, -1])])
def test_plans(lens, ids):
    rows = block(2).plan(lens, adapters=ids)[4]
    assert len(rows) == 2 and all(r.desc.n_adapters == 2 and r.desc.rank == 8 and r.desc.n_tokens == sum(lens) for r in rows)
    assert block(2).plan(lens)[4] is None


def test_what_a_step_refuses():
    """Tokens of another type or number, gradients of another shape: before anything is launched."""
    step = object.__new__(Tuning)
    step.d, step.table, step.block = 16, torch.zeros(9, 16, dtype=torch.float16), types.SimpleNamespace(dtype=0)
    plan = ([3, 4], None, None, None, None)
    good, dout, dtable = torch.zeros(7, dtype=torch.int32), torch.zeros(7, 16, dtype=torch.float16), torch.zeros(9, 16)
    for tokens in (good.long(), good[:6], torch.zeros(14, dtype=torch.int32)[::2], good[None]):
        with pytest.raises(ValueError):
            step.forward(tokens, plan)
        with pytest.raises(ValueError):
            step.backward(tokens, dout, plan, dtable)
    for wrong in ((dout[:6], dtable), (dout.float(), dtable), (dout, dtable.double()), (dout, dtable[:8]), (dout, torch.zeros(16, 9).t())):
        with pytest.raises(ValueError):
            step.backward(good, wrong[0], plan, wrong[1])


@pytest.mark.parametrize("d,dtype", [(64, B.BF16), (128, B.F16)])
def test_adapters_of_another_block(d, dtype):
    pool = Adapters(d, 2, 8, dtype=dtype, device="cpu")
    with pytest.raises(ValueError):
        TimeMix(64, 1, None, None, None, None, None, None, 1, 10, dtype=B.F16, adapters=pool)


@pytest.mark.parametrize("table", [torch.zeros(9, 16), torch.zeros(9, 8).half(), torch.zeros(16, 9).half().t(), torch.zeros(16).half()])
def test_tables_of_another_block(table):
    with pytest.raises(ValueError):
        Tuning(types.SimpleNamespace(d=16, dtype=B.F16, max_tokens=4), table)
