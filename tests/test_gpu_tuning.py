"""A tuning step end to end: embedding, time-mixing block with adapters and dropout, residual, and all gradients, against the same step in
binary64 on the CPU, differentiated by torch; the masks are the oracle's.

Bars.  As for the block without adapters (32 and 64 times 2^-11 of the largest value, there for eight roundings on the way and the norms
behind them); an adapter adds one more rounding to each of its five outputs and one to each gradient of their inputs, the residual one
forward and one back: 48 and 96 times.

What the first token of a sequence adds.  Its o is c v in each head, c = sum r u k, and the gradient `do` that comes through o's norm is orthogonal to o, so that
do . v, the factor of its dr = u k (do . v) and dk = u r (do . v), is 0 but for eps; in the block it is what rounding leaves of it.  do is rounded to fp16 (2^-11 of each
|do_c|), and it is orthogonal to the rounded o (2^-11 of each |o_c| = |c v_c|): either leaves up to 2^-11 sum |do_c v_c|.  do goes with 1 / c, and the block's c has eight
roundings in its factors, so is off by kappa = 8 2^-11 sum |r u k| / |c| of itself: together E = 2 (2 2^-11) sum |do v| / (1 - kappa), twice the two terms for what is left
of eps (its share of do . v goes with 1 / c as well), and no bar at all where kappa reaches 1.  `slack` takes E through the transposed matrices, mixes and the first norm with
magnitudes in the place of values: |dr| <= |u k| E, |dx_p| <= |dr| |W| and so on, to every gradient that these two reach."""
import numpy as np
import pytest

from oracle import tuning_oracle as TO

import gpu_util as G
from test_gpu_time_mix import close, params_of

pytestmark = pytest.mark.gpu
FORWARD, BACKWARD = 48 * 2.0 ** -11, 96 * 2.0 ** -11
D, HEADS, VOCAB = 256, 4, 50


def slack(block, dense, tokens, lens, ids, params, weights, masks, firsts):
    """What the first tokens add to the bars of the gradients, by name."""
    torch = G.torch_()
    ln_w, _, _, _, _, u = (p.detach() for p in params)
    out = {"table": torch.zeros(VOCAB, block.d, dtype=torch.float64), "ln weight": torch.zeros_like(ln_w), "ln bias": torch.zeros_like(ln_w), "u": torch.zeros_like(u)}
    for p in "rk":
        out[p, "a"], out[p, "b"] = (torch.zeros_like(t.detach()) for t in weights[p])
    for f in firsts:
        row, r, k, v, do = f["row"], f["r"], f["k"], f["v"], f["o"].grad[0].reshape(block.H, -1)
        c, size = (r * u * k).sum(-1), (r * u * k).abs().sum(-1)
        kappa = 8 * 2.0 ** -11 * size / c.abs()
        E = torch.where(kappa < 1, 4 * 2.0 ** -11 * (do * v).abs().sum(-1) / (1 - kappa), torch.inf)[:, None]
        d = {"r": ((u * k).abs() * E).reshape(-1), "k": ((u * r).abs() * E).reshape(-1)}
        da = 0.0
        for p, mu in zip("rk", f["mu"]):
            dx = d[p] @ dense[p].abs()
            if f["id"] >= 0:
                A, Bm = (t.detach()[f["id"]] for t in weights[p])
                scale, x = float(block.adapters.scales[f["id"]]), f["x"][p] * masks[p][row]
                g = scale * (d[p] @ Bm.abs())
                dx = dx + (g @ A.abs()) * masks[p][row]
                out[p, "a"][f["id"]] += g[:, None] * x.abs()
                out[p, "b"][f["id"]] += scale * d[p][:, None] * (A @ x).abs()
            da = da + mu * dx
        g, xhat = da * ln_w.abs(), f["xhat"].abs()
        out["ln weight"] += da * xhat
        out["ln bias"] += da
        out["u"] += (r * k).abs() * E
        if 0 <= tokens[row] < VOCAB:
            out["table"][tokens[row]] += f["rstd"] * (g + g.mean() + xhat * (g * xhat).mean())
    return out


def near(got, want, bar, what, more=0.0):
    got, want = got.detach().double().cpu().reshape(want.shape), want.detach()
    err = (got - want).abs() - bar * want.abs().max() - more
    assert not bool((err > 0).any()) and bool(torch_isfinite(got)), (what, float((got - want).abs().max() / want.abs().max()), float(err.max()))


def torch_isfinite(t):
    return G.torch_().isfinite(t).all()


def plain(block, dense, table, tokens, lens, ids, params, weights, masks, firsts):
    """The step in binary64.  weights: (a, b) by projection; masks: factors of the five inputs and of the block's output; firsts: takes what
    slack needs to know of each sequence's first token."""
    torch = G.torch_()
    ln_w, ln_b, h_w, h_b, w, u = params
    H, d = block.H, block.d
    live = torch.tensor([0 <= t < VOCAB for t in tokens])
    x = table[torch.tensor([t if 0 <= t < VOCAB else 0 for t in tokens])] * live[:, None]

    def norm(z, weight, bias, groups):
        y = z.reshape(z.shape[0], groups, -1)
        c = y - y.mean(-1, keepdim=True)
        return (c / torch.sqrt((c * c).mean(-1, keepdim=True) + block.eps)).reshape(z.shape) * weight + bias

    def project(p, v, rows, a):
        y = v @ dense[p].T
        if a < 0:
            return y
        A, Bm = weights[p]
        return y + float(block.adapters.scales[a]) * ((v * masks[p][rows]) @ A[a].T) @ Bm[a].T

    a = norm(x, ln_w, ln_b, 1)
    outs, first = [], 0
    for n, id_ in zip(lens, ids):
        if not n:
            continue
        rows = slice(first, first + n)
        s = a[rows]
        prev = torch.cat([torch.zeros_like(s[:1]), s[:-1]])
        proj, mus, mixed = [], [], {}
        for p, index, book in zip("rkvg", block.indices, block.codebooks):
            mus.append(book.cpu().view(torch.float16).view(-1, 2)[index.cpu().long()].reshape(-1).double())
            mix = mus[-1] * s + (1 - mus[-1]) * prev
            mixed[p] = mix.detach()[0]
            proj.append(project(p, mix, rows, id_))
        r, k, v = (t.reshape(n, H, -1) for t in proj[:3])
        S = torch.zeros(H, d // H, d // H, dtype=torch.float64)
        o = []
        for t in range(n):
            kv = k[t][:, :, None] * v[t][:, None, :]
            o.append((r[t][:, :, None] * (S + u[:, :, None] * kv)).sum(1))
            S = torch.exp(-w)[:, None, None] * S + kv
        o = torch.stack(o).reshape(n, d)
        o.retain_grad()
        z = norm(o, h_w, h_b, H)
        x0 = x.detach()[first]
        rstd = 1 / torch.sqrt(((x0 - x0.mean()) ** 2).mean() + block.eps)
        firsts.append(dict(row=first, id=id_, r=r.detach()[0], k=k.detach()[0], v=v.detach()[0], o=o, mu=mus[:2], x=mixed, rstd=rstd, xhat=(x0 - x0.mean()) * rstd))
        outs.append(project("o", torch.sigmoid(proj[3]) * z, rows, id_))
        first += n
    return x + torch.cat(outs) * masks["out"]


@pytest.fixture(scope="module")
def setup():
    torch = G.torch_()
    from paper_2505_03803_amd import binding as B, time_mix, tuning
    pool = time_mix.Adapters(D, 3, 16, p=0.25, seed=5)
    gen = torch.Generator().manual_seed(7)
    for p in pool.b:
        pool.b[p].copy_((torch.randn(pool.b[p].shape, generator=gen) * 0.1).half())
    pool.scales.copy_(torch.tensor([0.5, 1.0, 2.0]))
    block = time_mix.synthetic(D, HEADS, 3, 80, adapters=pool)
    dense = {p: B.dequant(m).cpu().double() for p, m in block.mats.items()}
    table = torch.randn(VOCAB, D, generator=gen).half().cuda()
    return block, dense, tuning.Tuning(block, table, p=0.1, seed=9)


def masks_of(step, T):
    """The factors that the oracle's generator gives for the step's seeds as they are."""
    torch = G.torch_()
    seeds = step.block.adapters.seeds.cpu().tolist()
    factors = lambda seed, p, call: torch.from_numpy(np.multiply(*TO.keep(seed, p, T, D, call)))  # noqa: E731
    masks = {p: factors(seeds[0], 0.25, i) for i, p in enumerate("rkvg")}
    return dict(masks, o=factors(seeds[1], 0.25, 0), out=factors(step.seed.cpu().tolist(), 0.1, 0))


@pytest.mark.parametrize("lens,ids", [([1], [2]), ([33], [0]), ([3, 0, 1, 20], [1, 0, -1, 1]), ([8, 8, 8], [2, -1, 0])])
def test_step(setup, lens, ids):
    torch = G.torch_()
    block, dense, step = setup
    T = sum(lens)
    rng = np.random.default_rng(T)
    tokens = rng.integers(0, 12, size=T)
    if T > 5:
        tokens[3] = -1                                     # padding inside a batch
    dev = torch.tensor(tokens, dtype=torch.int32, device="cuda")
    dout = torch.from_numpy(rng.standard_normal((T, D))).half()
    plan = step.plan(lens, ids)
    dtable = torch.full((VOCAB, D), 7.0, device="cuda")
    step.advance()
    masks = masks_of(step, T)
    table = step.table.cpu().double().requires_grad_()
    params = params_of(block)
    weights = {p: tuple(t[p].cpu().double().requires_grad_() for t in (block.adapters.a, block.adapters.b)) for p in "rkvgo"}
    firsts = []
    want = plain(block, dense, table, tokens, lens, ids, params, weights, masks, firsts)
    want.backward(dout.double())
    close(step.forward(dev, plan), want, FORWARD, "out")
    got = step.backward(dev, dout.cuda(), plan, dtable)
    more = slack(block, dense, tokens, lens, ids, params, weights, masks, firsts)
    near(got["table"], table.grad, BACKWARD, "table", more["table"])
    for name, g, p in zip(["ln weight", "ln bias", "heads weight", "heads bias", "w", "u"], [*got["ln"], *got["heads_norm"], got["w"], got["u"]], params):
        if T > 1 or name not in ("w", "u"):                # of a lone token both are nothing but rounding, as in the block's own test
            near(g, p.grad, BACKWARD, name, more.get(name, 0.0))
    for p in "rkvgo":
        for name, g, t in zip("ab", got["adapters"][p], weights[p]):
            grad = t.grad if t.grad is not None else torch.zeros_like(t)
            if T == 1 and p in "rk":
                continue                                   # r and k scale a lone token's o, which its norm takes out again
            if float(grad.abs().max()) == 0.0:
                assert float(g.abs().max()) == 0.0
            else:
                near(g, grad, BACKWARD, (p, name), more.get((p, name), 0.0))
    assert bool((got["table"][[v for v in range(VOCAB) if v not in tokens]] == 0.0).all())
    # added to what is there: the same sums once more
    again = step.backward(dev, dout.cuda(), plan, dtable.clone(), accumulate=True)
    assert torch.equal(again["table"], 2 * dtable)


def test_adapters_that_have_not_learnt_and_plans_without(setup):
    """B = 0, as adapters begin, or no adapter: the block's own bits."""
    torch = G.torch_()
    block, _, _ = setup
    x = torch.randn(24, D, device="cuda").half()
    bare = block.forward(x, block.plan([20, 4])).clone()
    none = block.forward(x, block.plan([20, 4], adapters=[-1, -1])).clone()
    assert torch.equal(bare, none)
    some = block.forward(x, block.plan([20, 4], adapters=[-1, 1])).clone()
    assert torch.equal(bare[:20], some[:20]) and not torch.equal(bare[20:], some[20:])
    kept = {p: t.clone() for p, t in block.adapters.b.items()}
    for t in block.adapters.b.values():
        t.zero_()
    fresh = block.forward(x, block.plan([20, 4], adapters=[0, 1], drop=True)).clone()
    for p, t in kept.items():
        block.adapters.b[p].copy_(t)
    assert torch.equal(bare, fresh)


def test_tokens_of_many_users_as_a_graph(setup):
    """Single tokens with an adapter each, captured and replayed, against the same tokens in one prompt for each user."""
    torch = G.torch_()
    block, _, _ = setup
    ids, steps = [2, 0, -1], 4
    x = torch.randn(3, steps, D, device="cuda").half()
    block.state.zero_(); block.last.zero_()
    want = torch.stack([block.forward(x[i], block.plan([steps], [i], adapters=[a])).clone() for i, a in enumerate(ids)])
    block.state.zero_(); block.last.zero_()
    token = torch.zeros(3, D, device="cuda").half()
    replay = block.capture(token, block.plan([1, 1, 1], [0, 1, 2], adapters=ids))
    for t in range(steps):
        token.copy_(x[:, t])
        close(replay().clone(), want[:, t], FORWARD, t)
