"""The multi-head time-mixing block end to end: norms, token-shift mixes, quantized projections, linear attention, gate, and the
gradients, against the same block in binary64 on the CPU (its gradients by torch's differentiation of the plain recurrence).

Bars.  Every intermediate is rounded to fp16 once (2^-11 of itself): a, mix, the weight fed to the matrix cores, projection, o, z,
gated, out is 8 roundings forward; the norms divide by a deviation whose own error is that of o, and the gate and the product of
three projections in o add up relative errors, so up to four times the plain count reaches an output: 32 x 2^-11 of the largest
value.  Backward meets as many roundings again on the way: 64 x 2^-11."""
import numpy as np
import pytest

from oracle import rwkvq_oracle as orc

import gpu_util as G

pytestmark = pytest.mark.gpu
FORWARD, BACKWARD = 32 * 2.0 ** -11, 64 * 2.0 ** -11


def close(got, want, bar, what):
    got, want = got.detach().double().cpu(), want.detach().double().cpu()
    err = float((got.reshape(want.shape) - want).abs().max() / want.abs().max())
    assert err <= bar, (what, err)


def plain(block, dense, x, lens, params, empty=True):
    """The block in binary64 with params = ln weight, bias, heads weight, bias, w, u; every sequence begins empty."""
    torch = G.torch_()
    ln_w, ln_b, h_w, h_b, w, u = params
    H, D, d = block.H, block.D, block.d

    def norm(z, weight, bias, groups):
        y = z.reshape(z.shape[0], groups, -1)
        c = y - y.mean(-1, keepdim=True)
        return (c / torch.sqrt((c * c).mean(-1, keepdim=True) + block.eps)).reshape(z.shape) * weight + bias

    a = norm(x, ln_w, ln_b, 1)
    outs, first = [], 0
    for n in lens:
        if not n:
            continue
        s = a[first:first + n]
        prev = torch.cat([torch.zeros_like(s[:1]), s[:-1]])
        proj = []
        for p, index, book in zip("rkvg", block.indices, block.codebooks):
            mu = book.cpu().view(torch.float16).view(-1, 2)[index.cpu().long()].reshape(-1).double()
            proj.append((mu * s + (1 - mu) * prev) @ dense[p].T)
        r, k, v = (t.reshape(n, H, D) for t in proj[:3])
        S = torch.zeros(H, D, D, dtype=torch.float64)
        o = []
        for t in range(n):
            kv = k[t][:, :, None] * v[t][:, None, :]
            o.append((r[t][:, :, None] * (S + u[:, :, None] * kv)).sum(1))
            S = torch.exp(-w)[:, None, None] * S + kv
        z = norm(torch.stack(o).reshape(n, d), h_w, h_b, H)
        outs.append((torch.sigmoid(proj[3]) * z) @ dense["o"].T)
        first += n
    return torch.cat(outs)


@pytest.fixture(scope="module")
def setup():
    torch = G.torch_()
    from paper_2505_03803_amd import binding as B, time_mix
    block = time_mix.synthetic(256, 4, 5, 80)
    dense = {p: B.dequant(m).cpu().double() for p, m in block.mats.items()}
    x = torch.from_numpy(np.random.default_rng(1).standard_normal((80, 256))).to(torch.float16)
    return block, dense, x


def params_of(block):
    return [t.cpu().double().requires_grad_() for t in (*block.ln, *block.heads_norm, block.w, block.u)]


@pytest.mark.parametrize("lens", [[1], [7], [70], [3, 0, 1, 20], [16, 16, 16, 16]])
def test_prompts(setup, lens):
    torch = G.torch_()
    block, dense, x = setup
    T = sum(lens)
    slots = [4, 0, 3, 1][:len(lens)]
    block.state.zero_(); block.last.zero_()
    got = block.forward(x[:T].cuda(), block.plan(lens, slots)).clone()
    close(got, plain(block, dense, x[:T].double(), lens, params_of(block)), FORWARD, lens)
    again = block.forward(x[:T].cuda(), block.plan(lens))            # empty sequences without slots: the same numbers
    assert torch.equal(got, again)


def test_tokens_behind_prompts_as_a_graph(setup):
    """Two prompts, then five tokens of each by a replayed graph, with eager work between the replays."""
    torch = G.torch_()
    block, dense, x = setup
    lens, steps = [9, 21], 5
    want = [plain(block, dense, x[40 * i:40 * i + n + steps].double(), [n + steps], params_of(block)) for i, n in enumerate(lens)]
    block.state.zero_(); block.last.zero_()
    block.forward(torch.cat([x[40 * i:40 * i + n] for i, n in enumerate(lens)]).cuda(), block.plan(lens, [2, 1]))
    token = torch.zeros(2, 256, dtype=torch.float16, device="cuda")
    replay = block.capture(token, block.plan([1, 1], [2, 1]))
    for t in range(steps):
        token.copy_(torch.stack([x[40 * i + n + t] for i, n in enumerate(lens)]))
        got = replay().clone()
        for i, n in enumerate(lens):
            close(got[i], want[i][n + t], FORWARD, (t, i))


@pytest.mark.parametrize("lens", [[1], [70], [3, 0, 1, 20]])
def test_gradients(setup, lens):
    torch = G.torch_()
    block, dense, x = setup
    T = sum(lens)
    dout = torch.from_numpy(np.random.default_rng(2).standard_normal((T, 256))).to(torch.float16)
    params, xs = params_of(block), x[:T].double().requires_grad_()
    plain(block, dense, xs, lens, params).backward(dout.double())
    plan, dx = block.plan(lens), x[:T].cuda()
    block.forward(dx, plan)
    got = block.backward(dx, dout.cuda(), plan)
    flat = [got["x"], *got["ln"], *got["heads_norm"], got["w"], got["u"]]
    names = ["x", "ln weight", "ln bias", "heads weight", "heads bias", "w", "u"]
    for name, g, p in zip(names, flat, [xs] + params):
        if name == "u" and lens == [1]:
            # A lone token's o is a multiple of v in each head, and the gradient behind a norm is orthogonal to the norm's input, so
            # that do . v, and with it the gradient of u, is 0 but for eps: what is left of it is the rounding of do.
            continue
        want = p.grad if p.grad is not None else torch.zeros_like(p)
        if float(want.abs().max()) == 0.0:                           # w of single tokens: no state meets a decay
            assert float(g.abs().max()) == 0.0, name
        else:
            close(g, want, BACKWARD, (lens, name))
