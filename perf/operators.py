"""What the operators of a multi-head RWKV block beside its projections are timed on: layer norm (forward and backward, whole
rows or a norm of its own for each head) and linear attention with a decay for each head (prompts, single tokens, backward).

    y_c    = (x_c - mean) / sqrt(var + eps) * weight_c + bias_c                           per row, or per head of a row
    out_t  = r_t (S_{t-1} + diag(u) k_t^T v_t),    S_t = exp(-w) S_{t-1} + k_t^T v_t        per sequence and head; S is head_dim x head_dim

Shapes are those of the repository's configurations (d = 4096 is 64 heads of 64, d = 5120 is 80) or drawn in between.  Decays and
the bonus are spread as for the repository's other block operators: w log-uniform over e^-5 .. e^1, u ~ N(0, 0.5).
"""
import math
import random

import torch

own = False

TYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
EPS = 1e-5


# ---- cases ------------------------------------------------------------------------------------------------------

def listed():
    return [
        # the norm in front of a projection while one user's text is generated: a launch's latency
        dict(name="norm_token", op="norm", M=1, groups=1, n=4096, x="f16"),
        # the same for a prompt of 2048 tokens, 14B-class width
        dict(name="norm_prompt", op="norm", M=2048, groups=1, n=5120, x="bf16"),
        # the norm of each of 64 heads behind attention, a ragged prompt
        dict(name="norm_heads", op="norm", M=333, groups=64, n=64, x="f16"),
        # tuning norm weights on binary32 activations of a width that no vector load divides
        dict(name="norm_grad_odd", op="norm_grad", M=777, groups=1, n=1023, x="f32"),
        # one training step's norm, 4 sequences of 2048 tokens
        dict(name="norm_grad_train", op="norm_grad", M=8192, groups=1, n=4096, x="bf16"),
        # one token for one user
        dict(name="step_one", op="step", seqs=1, heads=64, dim=64, x="f16"),
        # one token for each of 256 users, whose states lie in a pool
        dict(name="step_many", op="step", seqs=256, heads=64, dim=64, x="bf16"),
        # a short prompt
        dict(name="prompt_short", op="prompt", seqs=1, tokens=77, heads=64, dim=64, x="f16", ragged=False, fused=False),
        # prompts of sixteen users, each of its own length (one of them empty), r, k and v columns of one buffer; 14B-class width
        dict(name="prompt_ragged", op="prompt", seqs=16, tokens=4321, heads=80, dim=64, x="bf16", ragged=True, fused=True),
        # one long prompt
        dict(name="prompt_long", op="prompt", seqs=1, tokens=8192, heads=64, dim=64, x="bf16", ragged=False, fused=False),
        # gradients for a few ragged sequences, wide heads
        dict(name="grad_ragged", op="grad", seqs=5, tokens=1001, heads=16, dim=128, x="f16", ragged=True, fused=False),
        # one training step's attention, 4 sequences of 2048 tokens
        dict(name="grad_train", op="grad", seqs=4, tokens=8192, heads=64, dim=64, x="bf16", ragged=False, fused=False),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["norm", "norm", "norm_grad", "norm_grad", "step", "step", "prompt", "prompt", "grad", "grad"])
    x = rng.choice(["f16", "bf16"])
    if op.startswith("norm"):
        x = rng.choice([x, x, "f32"])
        groups = rng.choice([1, 1, 1, 16, 40, 64, 80])
        if groups == 1:
            n = rng.choice([_log(rng, 64, 16384), 8 * _log(rng, 8, 2048), 256 * _log(rng, 1, 64)])
        else:
            n = rng.choice([32, 64, 64, 128, 8 * rng.randint(2, 16), rng.randint(3, 128)])
        return dict(op=op, M=min(_log(rng, 1, 16384), 8192 * 4096 // (groups * n)), groups=groups, n=n, x=x)
    dim = rng.choice([32, 64, 64, 64, 128, 8 * rng.randint(2, 16)])
    heads = _log(rng, 2, 80)
    if op == "step":
        seqs = min(_log(rng, 1, 512), 256 * 64 * 64 * 64 // (heads * dim * dim))
        return dict(op=op, seqs=seqs, heads=heads, dim=dim, x=x)
    seqs = rng.choice([1, 1, _log(rng, 2, 32)])
    longest = (8192 if op == "prompt" else 4096) // (1 if seqs == 1 else 4)
    tokens = seqs * _log(rng, 16, longest) + rng.randint(0, seqs - 1)
    ragged = seqs > 1 and rng.random() < 0.7
    if not ragged:
        tokens -= tokens % seqs
    tokens = max(seqs, min(tokens, 8192 * 64 * 64 // (heads * dim) // seqs * seqs))
    return dict(op=op, seqs=seqs, tokens=tokens, heads=heads, dim=dim, x=x, ragged=ragged, fused=rng.random() < 0.3)


def _lengths(c):
    """The lengths of a case's sequences: alike, or ragged ones that add up to its tokens, the second one empty and the third a single token."""
    B, T = c["seqs"], c["tokens"]
    if not c["ragged"]:
        return [T // B] * B
    rng = random.Random("%d sequences, %d tokens" % (B, T))
    parts = [rng.expovariate(1.0) for _ in range(B)]
    parts = [0.0 if i == 1 or (i == 2 and B > 3) else min(p, 3.0) for i, p in enumerate(parts)]
    lens = [int(p / sum(parts) * (T - 1)) for p in parts]
    if B > 3:
        lens[2] = 1
    lens[0] += T - sum(lens)
    return lens


# ---- inputs -----------------------------------------------------------------------------------------------------

def prepare(case, seed):
    c = dict(case)
    t = TYPES[c["x"]]
    g = torch.Generator(device="cuda").manual_seed(seed)
    normal = lambda *shape: torch.randn(*shape, generator=g, device="cuda")  # noqa: E731
    s = {"case": c}
    if c["op"].startswith("norm"):
        M, n, wide = c["M"], c["n"], c["groups"] * c["n"]
        s["x"] = (normal(M, wide) * 1.5 + normal(1, wide)).to(t)                 # an offset and a spread of its own for each channel
        s["weight"], s["bias"] = 1.0 + 0.3 * normal(wide), 0.2 * normal(wide)
        s["y"] = torch.empty_like(s["x"])
        if c["op"] == "norm_grad":
            rows = s["x"].float().reshape(M, c["groups"], n)
            s["mean"] = rows.mean(-1)
            s["rstd"] = torch.rsqrt((rows - s["mean"][..., None]).square().mean(-1) + EPS)   # as the forward pass left them
            s["dy"] = normal(M, wide).to(t)
            s["dx"], s["dweight"], s["dbias"] = torch.empty_like(s["x"]), torch.empty(wide, device="cuda"), torch.empty(wide, device="cuda")
    else:
        B, H, D = c["seqs"], c["heads"], c["dim"]
        N = B if c["op"] == "step" else c["tokens"]
        wide = H * D
        rkv = normal(3, N, wide).mul_(torch.tensor([1.0, 0.5, 1.0], device="cuda")[:, None, None])
        if c.get("fused"):
            s["rkv"] = rkv.transpose(0, 1).to(t).reshape(N, 3 * wide)
            s["r"], s["k"], s["v"] = s["rkv"][:, :wide], s["rkv"][:, wide:2 * wide], s["rkv"][:, 2 * wide:]
        else:
            s["r"], s["k"], s["v"] = (p.to(t) for p in rkv)
        s["w"] = torch.exp(torch.rand(H, generator=g, device="cuda") * 6.0 - 5.0)
        s["u"] = 0.5 * normal(H, D)
        if c["op"] == "step":
            pool = B + B // 2
            s["slots"] = torch.randperm(pool, generator=g, device="cuda")[:B].to(torch.int32)
            s["state"], s["out"] = normal(pool, H, D, D), torch.empty(N, wide, dtype=t, device="cuda")
        else:
            lens = _lengths(c)
            s["longest"] = max(lens)
            s["offsets"] = torch.tensor([sum(lens[:i]) for i in range(B + 1)], dtype=torch.int32, device="cuda")
            s["state"] = normal(B, H, D, D)
            if c["op"] == "prompt":
                s["out"], s["state_out"] = torch.empty(N, wide, dtype=t, device="cuda"), torch.empty(B, H, D, D, device="cuda")
            else:
                s["dout"], s["dstate"] = normal(N, wide).to(t), 0.1 * normal(B, H, D, D)
                whole = torch.empty(N, 3 * wide, dtype=t, device="cuda") if c["fused"] else torch.empty(3, N, wide, dtype=t, device="cuda")
                s["dr"], s["dk"], s["dv"] = (whole[:, i * wide:(i + 1) * wide] for i in range(3)) if c["fused"] else whole
                s["dw"], s["du"], s["dstate_in"] = torch.empty(H, device="cuda"), torch.empty(H, D, device="cuda"), torch.empty(B, H, D, D, device="cuda")
    if own:
        _plan(s)
    return s


def _plan(s):
    """What a program keeps from call to call: the description of the sequences and the workspace."""
    from paper_2505_03803_amd import binding as B
    c = s["case"]
    size = 0
    s["type"] = B.DTYPES[c["x"]]
    if c["op"] == "norm_grad":
        size = B.rwkvq_layer_norm_backward_workspace_size(c["M"], c["groups"], c["n"])
    elif c["op"] == "step":
        s["heads"] = B.Heads(c["seqs"], c["seqs"], c["heads"], c["dim"], slots=s["slots"], n_slots=s["state"].shape[0])
        size = B.rwkvq_linear_attention_workspace_size(s["heads"])
    elif c["op"] in ("prompt", "grad"):
        row = s["r"].stride(0)
        s["heads"] = B.Heads(c["seqs"], c["tokens"], c["heads"], c["dim"], offsets=s["offsets"] if c["ragged"] else None,
                             r_stride=row, k_stride=row, v_stride=row)
        size = (B.rwkvq_linear_attention_workspace_size if c["op"] == "prompt" else B.rwkvq_linear_attention_backward_workspace_size)(s["heads"])
    s["workspace"] = torch.empty(max(size, 16), dtype=torch.uint8, device="cuda")


# ---- one pass ---------------------------------------------------------------------------------------------------

def run(s):
    return (_own if own else _plain)[s["case"]["op"]](s)


def _own_norm(s):
    from paper_2505_03803_amd import binding as B
    c = s["case"]
    B.rwkvq_layer_norm(s["x"], s["type"], c["M"], c["groups"], c["n"], s["weight"], s["bias"], EPS, s["y"])
    return s["y"]


def _own_norm_grad(s):
    from paper_2505_03803_amd import binding as B
    c = s["case"]
    B.rwkvq_layer_norm_backward(s["dy"], s["x"], s["type"], c["M"], c["groups"], c["n"], s["weight"], s["mean"], s["rstd"], s["dx"], s["dweight"],
                                s["dbias"], s["workspace"])
    return s["dx"], s["dweight"], s["dbias"]


def _own_step(s):
    from paper_2505_03803_amd import binding as B
    B.rwkvq_linear_attention(s["heads"], s["r"], s["k"], s["v"], s["type"], s["w"], s["u"], s["state"], s["state"], s["out"], s["workspace"])
    return s["out"], s["state"]


def _own_prompt(s):
    from paper_2505_03803_amd import binding as B
    B.rwkvq_linear_attention(s["heads"], s["r"], s["k"], s["v"], s["type"], s["w"], s["u"], s["state"], s["state_out"], s["out"], s["workspace"])
    return s["out"], s["state_out"]


def _own_grad(s):
    from paper_2505_03803_amd import binding as B
    B.rwkvq_linear_attention_backward(s["heads"], s["r"], s["k"], s["v"], s["dout"], s["type"], s["w"], s["u"], s["state"], s["dstate"],
                                      s["dr"], s["dk"], s["dv"], s["dw"], s["du"], s["dstate_in"], s["workspace"])
    return s["dr"], s["dk"], s["dv"], s["dw"], s["du"], s["dstate_in"]


_own = {"norm": _own_norm, "norm_grad": _own_norm_grad, "step": _own_step, "prompt": _own_prompt, "grad": _own_grad}


# The plain forms: binary32 throughout, one rounding at the end.

def _plain_norm(s):
    c = s["case"]
    x = s["x"].float().reshape(c["M"], c["groups"], c["n"])
    d = x - x.mean(-1, keepdim=True)
    y = d * torch.rsqrt(d.square().mean(-1, keepdim=True) + EPS)
    return (y.reshape(c["M"], -1) * s["weight"] + s["bias"]).to(s["x"].dtype)


def _plain_norm_grad(s):
    c = s["case"]
    shape = c["M"], c["groups"], c["n"]
    xhat = (s["x"].float().reshape(shape) - s["mean"][..., None]) * s["rstd"][..., None]
    dy = s["dy"].float()
    g = (dy * s["weight"]).reshape(shape)
    dx = s["rstd"][..., None] * (g - g.mean(-1, keepdim=True) - xhat * (g * xhat).mean(-1, keepdim=True))
    return dx.reshape(c["M"], -1).to(s["x"].dtype), (dy * xhat.reshape(c["M"], -1)).sum(0), dy.sum(0)


def _plain_step(s):
    c = s["case"]
    r, k, v = (s[p].float().reshape(c["seqs"], c["heads"], c["dim"]) for p in "rkv")
    slots = s["slots"].long()
    S = s["state"][slots]
    kv = k[..., :, None] * v[..., None, :]
    out = (r[..., :, None] * (S + s["u"][..., None] * kv)).sum(-2)
    s["state"][slots] = torch.exp(-s["w"])[:, None, None] * S + kv
    return out.reshape(c["seqs"], -1).to(s["r"].dtype), s["state"]


def _padded(s, wide=("r", "k", "v")):
    """The rows of each sequence as [sequence, head, token, channel], with zeros behind its end; the rows' places and the lengths."""
    c = s["case"]
    first = s["offsets"][:-1].long()
    lens = s["offsets"][1:].long() - first
    t = torch.arange(s["longest"], device="cuda")
    live = t < lens[:, None]
    at = torch.where(live, first[:, None] + t, 0)
    rows = [(s[p].float()[at] * live[..., None]).reshape(c["seqs"], -1, c["heads"], c["dim"]).transpose(1, 2) for p in wide]
    return rows, at[live], live, lens


def _decay(s, T):
    """exp(-(t - 1 - i) w) for the pairs t > i of each head, and t - 1 - i."""
    t = torch.arange(T, device="cuda", dtype=torch.float32)
    lag = t[:, None] - 1.0 - t[None, :]
    decay = torch.exp(lag.clamp(min=0.0) * -s["w"][:, None, None])
    return decay.mul_(lag >= 0.0), lag, t


def _rows(x, live, dtype):
    """[sequence, head, token, channel] back to rows of tokens, those behind a sequence's end left out."""
    return x.transpose(1, 2).flatten(2)[live].to(dtype)


def _plain_prompt(s):
    (r, k, v), _, live, lens = _padded(s)
    decay, _, t = _decay(s, s["longest"])
    w = s["w"][:, None]
    past = torch.exp(-t * w)[..., None]                                                  # weight of the state in front
    left = torch.exp(-(lens[:, None, None] - 1.0 - t).clamp(min=0.0) * w)[..., None]      # of a token in the state behind
    A = (r @ k.transpose(-1, -2)).mul_(decay)
    out = A @ v + (r * s["u"][:, None] * k).sum(-1, keepdim=True) * v + past * (r @ s["state"])
    state = torch.exp(-lens[:, None] * s["w"])[..., None, None] * s["state"] + (left * k).transpose(-1, -2) @ v
    return _rows(out, live, s["r"].dtype), state


def _plain_grad(s):
    (r, k, v, do), _, live, lens = _padded(s, ("r", "k", "v", "dout"))
    decay, lag, t = _decay(s, s["longest"])
    w, u, S, dS = s["w"][:, None], s["u"][:, None], s["state"], s["dstate"]
    past = torch.exp(-t * w)[..., None]
    behind = (lens[:, None, None] - 1.0 - t).clamp(min=0.0)
    left = torch.exp(-behind * w)[..., None]
    whole = torch.exp(-lens[:, None] * s["w"])[..., None, None]
    A = (r @ k.transpose(-1, -2)).mul_(decay)
    X = do @ v.transpose(-1, -2)
    dw = (A * X).mul_(lag).sum((-1, -2))
    X.mul_(decay)
    now = (do * v).sum(-1, keepdim=True)
    from_state, to_state = past * (do @ S.transpose(-1, -2)), left * (v @ dS.transpose(-1, -2))
    dr = X @ k + now * u * k + from_state
    dk = X.transpose(-1, -2) @ r + now * u * r + to_state
    dv = A.transpose(-1, -2) @ do + (r * u * k).sum(-1, keepdim=True) * do + left * (k @ dS)
    dw = dw + (t * (from_state * r).sum(-1)).sum(-1) + (behind * (to_state * k).sum(-1)).sum(-1) + lens[:, None] * (whole * S * dS).sum((-1, -2))
    return (_rows(dr, live, s["r"].dtype), _rows(dk, live, s["r"].dtype), _rows(dv, live, s["r"].dtype), -dw.sum(0), (r * k * now).sum((0, 2)),
            whole * dS + (past * r).transpose(-1, -2) @ do)


_plain = {"norm": _plain_norm, "norm_grad": _plain_norm_grad, "step": _plain_step, "prompt": _plain_prompt, "grad": _plain_grad}


# ---- what a pass cannot do without ------------------------------------------------------------------------------

def work(c):
    size = 4 if c["x"] == "f32" else 2
    if c["op"].startswith("norm"):
        wide = c["groups"] * c["n"]
        if c["op"] == "norm":
            return {"bytes": 2 * c["M"] * wide * size + 8 * wide, "flops": 8 * c["M"] * wide}
        return {"bytes": 3 * c["M"] * wide * size + 12 * wide + 8 * c["M"] * c["groups"], "flops": 14 * c["M"] * wide}
    H, D = c["heads"], c["dim"]
    if c["op"] == "step":
        return {"bytes": c["seqs"] * H * (8 * D * D + 4 * D * size), "flops": c["seqs"] * H * 5 * D * D}
    # token by token a state takes D x D products for the output and as many for its update
    if c["op"] == "prompt":
        return {"bytes": 4 * c["tokens"] * H * D * size + 8 * c["seqs"] * H * D * D, "flops": 5 * c["tokens"] * H * D * D}
    return {"bytes": 7 * c["tokens"] * H * D * size + 12 * c["seqs"] * H * D * D, "flops": 12 * c["tokens"] * H * D * D}


# ---- the definition in 64 bits ----------------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    return _exact_norm(s) if case["op"].startswith("norm") else _exact_attention(s)


def _exact_norm(s):
    c = s["case"]
    rows = s["x"].double().reshape(-1, c["n"])
    var, mean = torch.var_mean(rows, dim=1, unbiased=False, keepdim=True)
    sigma = torch.sqrt(var + EPS)
    gain = s["weight"].double().reshape(1, c["groups"], c["n"]).expand(c["M"], -1, -1).reshape(-1, c["n"])
    if c["op"] == "norm":
        shift = s["bias"].double().reshape(1, c["groups"], c["n"]).expand(c["M"], -1, -1).reshape(-1, c["n"])
        return ((rows - mean) / sigma * gain + shift).reshape(c["M"], -1)
    dy = s["dy"].double().reshape(-1, c["n"])
    z = (rows - mean) / sigma
    # the gradient of z has its parts along the ones and along z taken out, over sigma
    g = dy * gain
    dx = (g - g.sum(1, keepdim=True) / c["n"] - z * (g * z).sum(1, keepdim=True) / c["n"]) / sigma
    return dx.reshape(c["M"], -1), (dy * z).reshape(c["M"], -1).sum(0), dy.reshape(c["M"], -1).sum(0)


def _exact_attention(s):
    """Token by token, the tokens of all sequences that are long enough at once; the gradient of w by carrying the state's derivative along."""
    c = s["case"]
    B, H, D = c["seqs"], c["heads"], c["dim"]
    grad = c["op"] == "grad"
    rows = {p: s[p].double().reshape(-1, H, D) for p in ("r", "k", "v", "dout") if p in s}
    lam, u = torch.exp(-s["w"].double())[:, None, None], s["u"].double()
    lens = [1] * B if c["op"] == "step" else _lengths(c)
    begin = [sum(lens[:b]) for b in range(B)]
    order = sorted(range(B), key=lambda b: -lens[b])                       # long ones first: those that have a token t are the first few
    where = torch.tensor([begin[b] for b in order], device="cuda")
    slots = s["slots"].long() if c["op"] == "step" else torch.arange(B, device="cuda")
    slots = slots[torch.tensor(order, device="cuda")]
    count = [sum(n > t for n in lens) for t in range(max(lens))]
    S = s["state"].double()[slots]
    out = torch.zeros_like(rows["r"])
    if grad:
        dr, dk, dv = (torch.zeros_like(out) for _ in range(3))
        Z, dw = torch.zeros_like(S), torch.zeros(H, dtype=torch.float64, device="cuda")      # Z: derivative of S by -w
    for t, m in enumerate(count):
        at = where[:m] + t
        r, k, v = (rows[p][at] for p in "rkv")
        kv = k[..., :, None] * v[..., None, :]
        if grad:
            do = rows["dout"][at]
            dr[at] = ((S[:m] + u[..., None] * kv) @ do[..., None])[..., 0]
            dw -= (r * (Z[:m] @ do[..., None])[..., 0]).sum((0, 2))
            Z[:m] = lam * (Z[:m] + S[:m])
        else:
            out[at] = (r[..., None, :] @ (S[:m] + u[..., None] * kv))[..., 0, :]
        S[:m] = lam * S[:m] + kv
    if not grad:
        state = s["state"].double()
        state[slots] = S
        return out.reshape(-1, H * D), state
    G = s["dstate"].double()[slots]
    dw -= (G * Z).sum((0, 2, 3))
    du = torch.zeros_like(u)
    for t in reversed(range(len(count))):
        m = count[t]
        at = where[:m] + t
        r, k, v, do = (rows[p][at] for p in ("r", "k", "v", "dout"))
        now = (do * v).sum(-1, keepdim=True)
        dk[at] = (G[:m] @ v[..., None])[..., 0] + now * u * r
        dv[at] = (k[..., None, :] @ G[:m])[..., 0, :] + (r * u * k).sum(-1, keepdim=True) * do
        du += (r * k * now).sum(0)
        G[:m] = lam * G[:m] + r[..., :, None] * do[..., None, :]
    back = torch.empty_like(G)
    back[slots] = G
    return dr.reshape(-1, H * D), dk.reshape(-1, H * D), dv.reshape(-1, H * D), dw, du, back
