"""CPU-side check of a plan's form: that of a block without adapters has four parts, and of one with them the rows of the adapters as well."""
from test_tuning_plan import block


def test_parts():
    lens, slots, heads, workspace = block(0).plan([3, 4], [1, 0])
    assert (lens, slots, heads.desc.n_seqs, heads.desc.n_tokens) == ([3, 4], [1, 0], 2, 7) and workspace.numel() >= 16
    assert len(block(2).plan([3, 4])) == 5 and len(block(2).plan([3, 4], adapters=[1, -1])[4]) == 2
