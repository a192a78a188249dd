"""CPU-side checks of the time-mixing block's plans: sequences that its buffers or its pool of states do not hold are refused."""
import pytest

from paper_2505_03803_amd.time_mix import TimeMix


@pytest.fixture
def block():
    b = object.__new__(TimeMix)                            # what plan() looks at, without a GPU
    b.H, b.D, b.max_tokens, b.n_slots, b.device = 2, 64, 40, 5, "cpu"
    return b


# a slot outside the pool, also one that Python would count from its end; one that two sequences share; one too many; one too few
@pytest.mark.parametrize("lens,slots", [([1, 1], [0, -1]), ([1, 1], [5, 0]), ([3, 4], [2, 2]), ([3, 4], [1, 1, 2]), ([3, 4], [1]), ([1], [2 ** 31])])
def test_slots_that_are_refused(block, lens, slots):
    with pytest.raises(ValueError):
        block.plan(lens, slots)


@pytest.mark.parametrize("lens", [[41], [20, 21], [-1, 5]])
def test_lengths_that_are_refused(block, lens):
    with pytest.raises(ValueError):
        block.plan(lens)


@pytest.mark.parametrize("lens,slots", [([1, 1], [0, 4]), ([40], [3]), ([3, 0, 5], [4, 0, 2]), ([20, 20], None)])
def test_plans(block, lens, slots):
    assert block.plan(lens, slots)[0] == lens
