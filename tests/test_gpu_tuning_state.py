"""What a block and a tuning step keep between a forward call and its gradients: masks and tokens; and what
the table's gradient is summed from."""
import numpy as np
import pytest

from oracle import tuning_oracle as TO

import gpu_util as G

pytestmark = pytest.mark.gpu
torch = G.torch_()
D, HEADS, VOCAB = 256, 4, 40


def pool_of(seed):
    from paper_2505_03803_amd import time_mix
    pool = time_mix.Adapters(D, 2, 8, p=0.4, seed=seed)
    gen = torch.Generator().manual_seed(seed)
    for p in pool.b:
        pool.b[p].copy_((torch.randn(pool.b[p].shape, generator=gen) * 0.1).half())
    return pool


def block_of(pool, seed=0):
    from paper_2505_03803_amd import time_mix
    return time_mix.synthetic(D, HEADS, 2, 60, seed=seed, adapters=pool)


def flat(grads):
    """Every tensor of a dictionary of gradients, by name."""
    out = {}
    for name, g in grads.items():
        if isinstance(g, dict):
            out.update({(name, *((k,) if not isinstance(k, tuple) else k)): v for k, v in flat(g).items()})
        elif isinstance(g, tuple):
            out.update({(name, i): v for i, v in enumerate(g)})
        else:
            out[name] = g
    return {k: v.clone() for k, v in out.items()}


def same(a, b):
    assert a.keys() == b.keys()
    for name in a:
        assert torch.equal(a[name], b[name]), name


def test_gradients_of_a_block_have_the_masks_of_their_call():
    """Also where the numbers of the next call are set in between, by a step or by another block of the pool."""
    pool = pool_of(3)
    block, other = block_of(pool), block_of(pool, 1)
    torch.manual_seed(1)
    x, dout = torch.randn(30, D, device="cuda").half(), torch.randn(30, D, device="cuda").half()
    plan, beside = block.plan([20, 10], adapters=[0, 1], drop=True), other.plan([30], adapters=[1], drop=True)
    first = block.forward(x, plan).clone()
    want = flat(block.backward(x, dout, plan))
    pool.advance()
    same(want, flat(block.backward(x, dout, plan)))
    out = block.forward(x, plan).clone()
    assert not torch.equal(out, first)                     # other masks
    want = flat(block.backward(x, dout, plan))
    for _ in range(2):
        other.forward(x, beside)
        pool.advance()
    same(want, flat(block.backward(x, dout, plan)))


def test_gradients_behind_a_replayed_block_have_its_masks():
    pool = pool_of(4)
    block, plain = block_of(pool), block_of(pool)
    torch.manual_seed(2)
    x, dout = torch.randn(30, D, device="cuda").half(), torch.randn(30, D, device="cuda").half()
    plan, eager = block.plan([30], adapters=[1], drop=True), plain.plan([30], adapters=[1], drop=True)
    replay = block.capture(x, plan)
    for i in range(3):
        x.normal_()
        pool.advance()
        out = replay()
        assert torch.equal(out, plain.forward(x, eager))
        want = flat(plain.backward(x, dout, eager))
        pool.advance()
        same(want, flat(block.backward(x, dout, plan)))


@pytest.fixture(scope="module")
def step():
    from paper_2505_03803_amd import tuning
    torch.manual_seed(3)
    return tuning.Tuning(block_of(pool_of(5)), torch.randn(VOCAB, D).half().cuda(), p=0.3, seed=8)


def batch(T, seed):
    rng = np.random.default_rng(seed)
    return torch.tensor(rng.integers(-1, VOCAB, size=T), dtype=torch.int32, device="cuda"), torch.from_numpy(rng.standard_normal((T, D))).half().cuda()


def test_gradients_of_a_step_have_the_masks_of_their_call(step):
    tokens, dout = batch(30, 0)
    plan, dtable = step.plan([11, 19], [1, 0]), torch.empty(VOCAB, D, device="cuda")
    step.forward(tokens, plan)
    want = flat(step.backward(tokens, dout, plan, dtable))
    step.advance()
    same(want, flat(step.backward(tokens, dout, plan, dtable)))
    p, step.p = step.p, 0.0
    same(want, flat(step.backward(tokens, dout, plan, dtable)))
    step.p = p


def test_gradients_of_another_batch_are_refused(step):
    tokens, dout = batch(30, 1)
    others, _ = batch(30, 2)
    plan, dtable = step.plan([30], [1]), torch.empty(VOCAB, D, device="cuda")
    step.forward(tokens, plan)
    step.forward(others, plan)
    with pytest.raises(ValueError):
        step.backward(tokens, dout, plan, dtable)
    step.backward(others, dout, plan, dtable)


@pytest.mark.parametrize("added", [False, True])
def test_table_gradients_are_sums_of_binary32(step, added):
    """dx + dout is binary32, one rounding of 2^-24 in each term: with those of the sum, of the product and of what is added (count + 3) 2^-24."""
    tokens, dout = batch(50, 4)
    plan = step.plan([30, 20], [0, 1])
    step.forward(tokens, plan)
    before = torch.randn(VOCAB, D, device="cuda") if added else torch.zeros(VOCAB, D, device="cuda")
    dtable = before.clone()
    step.backward(tokens, dout, plan, dtable, accumulate=added)
    dx = step.block.backward(step.x[:50], step.dy[:50], plan)["x"]
    terms = dx.cpu().double().numpy() + dout.cpu().double().numpy()
    want, size, count = TO.embedding_backward(tokens.tolist(), terms, VOCAB)
    old = before.cpu().double().numpy()
    bar = 2.0 ** -24 * (count[:, None] + 3) * (size + np.abs(old))
    err = np.abs(dtable.cpu().double().numpy() - want - old)
    assert (err <= bar).all(), float((err / np.maximum(bar, 1e-300)).max())


def test_plans_without_adapters_have_no_gradients_of_them(step):
    block = step.block
    x, dout = torch.randn(30, D, device="cuda").half(), torch.randn(30, D, device="cuda").half()
    for adapters, names in ((None, {"x", "ln", "heads_norm", "w", "u"}), ([1], {"x", "ln", "heads_norm", "w", "u", "adapters"})):
        plan = block.plan([30], adapters=adapters)
        block.forward(x, plan)
        assert set(block.backward(x, dout, plan)) == names
