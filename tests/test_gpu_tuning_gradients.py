"""Gradients of a tuning step to which the first tokens of the sequences add nothing from outside: what their gradient is, rounding for the most part, is what the
bars of test_gpu_tuning.py make room for, without a limit where a head's sum of r u k nearly cancels.  Here every gradient has the fixed bar, 96 times 2^-11 of its
largest value: dout is 0 in those rows, and what comes back to them through the state and the token shift is a gradient like any other."""
import numpy as np
import pytest

import gpu_util as G
from test_gpu_time_mix import params_of
from test_gpu_tuning import BACKWARD, D, VOCAB, masks_of, near, plain, setup  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("lens,ids", [([33], [0]), ([3, 0, 1, 20], [1, 0, -1, 1]), ([8, 8, 8], [2, 1, 0]), ([2, 31, 2], [0, 2, 2])])
def test_gradients_without_first_tokens(setup, lens, ids):  # noqa: F811
    torch = G.torch_()
    block, dense, step = setup
    T = sum(lens)
    rng = np.random.default_rng(T + len(lens))
    tokens = rng.integers(0, 12, size=T)
    dev = torch.tensor(tokens, dtype=torch.int32, device="cuda")
    dout = torch.from_numpy(rng.standard_normal((T, D))).half()
    dout[[f for f, n in zip(np.concatenate([[0], np.cumsum(lens)]), lens) if n]] = 0
    plan = step.plan(lens, ids)
    step.advance()
    masks = masks_of(step, T)
    table = step.table.cpu().double().requires_grad_()
    params = params_of(block)
    weights = {p: tuple(t[p].cpu().double().requires_grad_() for t in (block.adapters.a, block.adapters.b)) for p in "rkvgo"}
    plain(block, dense, table, tokens, lens, ids, params, weights, masks, []).backward(dout.double())
    step.forward(dev, plan)
    got = step.backward(dev, dout.cuda(), plan, torch.empty(VOCAB, D, device="cuda"))
    pairs = [("table", got["table"], table.grad)]
    pairs += list(zip(["ln weight", "ln bias", "heads weight", "heads bias", "w", "u"], [*got["ln"], *got["heads_norm"], got["w"], got["u"]],
                      [p.grad for p in params]))
    for p in "rkvgo":
        pairs += [((p, name), g, t.grad) for name, g, t in zip("ab", got["adapters"][p], weights[p])]
    for name, g, want in pairs:
        assert bool(torch.isfinite(want).all()) and float(want.abs().max()) > 0.0, name
        near(g, want, BACKWARD, name)
