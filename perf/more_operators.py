"""What the operators that tuning takes around frozen quantized matrices are timed on: dropout whose mask is never stored, embedding
lookup with its gradient, and low-rank adapters of many requests beside a shared projection (prompts, single tokens, gradients).

    y_tc   = base_tc + keep_tc x_tc / (1 - p)                                 keep from a counter-based generator
    out_t  = scale table[token_t],      dtable_v = sum of scale dout_t over the t with token_t = v
    h_t    = A_a drop(x_t),   y_t = base_t + s_a B_a h_t                      a: the adapter of t's sequence, maybe none
    g_t    = s_a B_a^T dy_t,  dx_t = base_t + drop(A_a^T g_t),  dA_a = sum of g_t drop(x_t)^T,  dB_a = sum of s_a dy_t h_t^T

The generator is Philox 4x32-10 (Salmon, Moraes, Dror and Shaw, "Parallel random numbers: as easy as 1, 2, 3", 2011) with the counter
(column / 8, row, call) and the seed as its key: eight numbers of 16 bits for eight columns, dropped where below 65536 p.

Shapes are those of the repository's configurations (d = 4096 and 5120, the 4096 x 14336 of a feed-forward key) or drawn in between.  Tokens
are spread as words are, the i-th most frequent with a probability of about 1 / i, with identifiers in no order of frequency.
"""
import math
import random

import numpy as np
import torch

own = False

TYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}


# ---- cases ------------------------------------------------------------------------------------------------------

def listed():
    return [
        # the row of one user's token while text is generated: a launch's latency
        dict(name="embed_token", op="embed", tokens=1, vocab=65536, d=4096, table="f16", x="f16", scale=1.0, padded=False),
        # the rows of sixteen users' prompts, 14B-class width, scaled by the root of the width
        dict(name="embed_prompts", op="embed", tokens=4321, vocab=65536, d=5120, table="bf16", x="bf16", scale=71.55417527999327, padded=False),
        # tuning a small table of a width that no vector load divides, a padded batch; added to the gradient of the batch before
        dict(name="embed_grad_odd", op="embed_grad", tokens=777, vocab=5003, d=1023, x="f32", scale=1.0, padded=True, added=True),
        # one training step's gradient of a whole table, 4 sequences of 2048 tokens
        dict(name="embed_grad_train", op="embed_grad", tokens=8192, vocab=65536, d=4096, x="bf16", scale=1.0, padded=False, added=False),
        # dropout in front of a projection, a short sequence
        dict(name="drop_short", op="drop", M=77, n=4096, x="f16", p=0.1, base=False),
        # dropout of a block's output, added to the residual stream, one training step
        dict(name="drop_train", op="drop", M=8192, n=4096, x="bf16", p=0.1, base=True),
        # one token of one user, whose adapter sits beside the four projections of time mixing
        dict(name="adapter_token", op="adapter", seqs=1, tokens=1, adapters=3, mats=4, rank=16, K=4096, N=4096, x="f16", y="f16", p=0.0, ragged=False),
        # one token for each of 256 users of 64 adapters, the same four projections
        dict(name="adapter_users", op="adapter", seqs=256, tokens=256, adapters=64, mats=4, rank=16, K=4096, N=4096, x="bf16", y="bf16", p=0.0,
             ragged=False),
        # prompts of sixteen users (one of them empty) with seven adapters, some without one, beside a feed-forward key
        dict(name="adapter_prompts", op="adapter", seqs=16, tokens=4321, adapters=7, mats=1, rank=32, K=4096, N=14336, x="bf16", y="bf16", p=0.0,
             ragged=True),
        # the forward pass of one training step, 4 sequences of 2048 tokens, dropout in front of the adapter
        dict(name="adapter_train", op="adapter", seqs=4, tokens=8192, adapters=1, mats=1, rank=64, K=4096, N=4096, x="bf16", y="bf16", p=0.05,
             ragged=False),
        # gradients for a few ragged sequences of three adapters beside two projections of an odd shape
        dict(name="adapter_grad_ragged", op="adapter_grad", seqs=5, tokens=1001, adapters=3, mats=2, rank=8, K=2048, N=1000, x="f16", p=0.0, ragged=True),
        # the backward pass of the training step
        dict(name="adapter_grad_train", op="adapter_grad", seqs=4, tokens=8192, adapters=1, mats=1, rank=64, K=4096, N=4096, x="bf16", p=0.05,
             ragged=False),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["embed", "embed_grad", "embed_grad", "drop", "adapter", "adapter", "adapter", "adapter_grad", "adapter_grad"])
    x = rng.choice(["f16", "bf16"])
    width = rng.choice([1024, 2048, 4096, 4096, 5120, 8 * _log(rng, 8, 1024)])
    if op.startswith("embed"):
        x = rng.choice([x, x, "f32"])
        d = rng.choice([width, width, rng.randint(1, 5000)])
        vocab = rng.choice([65536, 256, _log(rng, 300, 65536)])
        tokens = min(_log(rng, 1, 16384), 8192 * 4096 // d)
        vocab = min(vocab, 65536 * 4096 // d)
        c = dict(op=op, tokens=tokens, vocab=vocab, d=d, x=x, scale=rng.choice([1.0, math.sqrt(d)]), padded=rng.random() < 0.3)
        if op == "embed":
            c["table"] = rng.choice([x, x, "f32"])
        else:
            c["added"] = rng.random() < 0.5
        return c
    if op == "drop":
        x = rng.choice([x, x, "f32"])
        n = rng.choice([width, width, rng.randint(1, 20000)])
        return dict(op=op, M=min(_log(rng, 1, 8192), 8192 * 4096 // n), n=n, x=x, p=rng.choice([0.0, 0.05, 0.1, 0.5]), base=rng.random() < 0.5)
    K, N = width, rng.choice([width, 1024, 4096, 8 * _log(rng, 8, 1792)])
    rank = rng.choice([8, 16, 16, 32, 64, 8 * rng.randint(1, 16)])
    mats = rng.choice([1, 1, 2, 4])
    seqs = rng.choice([1, 1, 4, _log(rng, 2, 256)])
    longest = max(1, min(8192, 8192 * 4096 * 64 // (mats * max(K, N) * max(rank, 64))) // seqs)
    tokens = seqs * (1 if op == "adapter" and rng.random() < 0.3 else _log(rng, 1, longest)) + rng.randint(0, seqs - 1)
    ragged = seqs > 1 and tokens > 2 * seqs and rng.random() < 0.7
    if not ragged:
        tokens -= tokens % seqs
    c = dict(op=op, seqs=seqs, tokens=tokens, adapters=_log(rng, 1, 64 if op == "adapter" else 8), mats=mats, rank=rank, K=K, N=N, x=x,
             p=rng.choice([0.0, 0.0, 0.05, 0.1]), ragged=ragged)
    if op == "adapter":
        c["y"] = rng.choice([x, x, "f32"])
    return c


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


def _ids(c):
    """The adapter of each sequence: every adapter as often as any other, in no order; of more than four sequences the last one has none."""
    ids = [b % c["adapters"] for b in range(c["seqs"])]
    random.Random("%d sequences, %d adapters" % (c["seqs"], c["adapters"])).shuffle(ids)
    if c["seqs"] > 4:
        ids[-1] = -1
    return ids


def _tokens(c):
    """Identifiers of a case's tokens on the host; of a padded batch the last eighth is padding, -1."""
    rng = np.random.default_rng([c["tokens"], c["vocab"], c["d"]])
    rank = np.floor(np.exp(rng.random(c["tokens"]) * np.log(c["vocab"] + 1.0))).astype(np.int64) - 1
    tokens = rng.permutation(c["vocab"])[np.clip(rank, 0, c["vocab"] - 1)]
    if c["padded"]:
        tokens[c["tokens"] - c["tokens"] // 8:] = -1
    return tokens


# ---- inputs -----------------------------------------------------------------------------------------------------

def prepare(case, seed):
    c = dict(case)
    t = TYPES[c["x"]]
    g = torch.Generator(device="cuda").manual_seed(seed)
    normal = lambda *shape: torch.randn(*shape, generator=g, device="cuda")  # noqa: E731
    s = {"case": c}
    if c["op"].startswith("embed"):
        order = torch.randperm(c["vocab"], generator=g, device="cuda")              # other tokens for another seed
        tokens = torch.from_numpy(_tokens(c)).cuda()
        s["tokens"] = torch.where(tokens >= 0, order[tokens.clamp(min=0)], -1).to(torch.int32)
        if c["op"] == "embed":
            s["table"] = (0.02 * normal(c["vocab"], c["d"])).to(TYPES[c["table"]])
            s["out"] = torch.empty(c["tokens"], c["d"], dtype=t, device="cuda")
        else:
            s["dout"] = normal(c["tokens"], c["d"]).to(t)
            s["dtable"] = normal(c["vocab"], c["d"]) if c["added"] else torch.empty(c["vocab"], c["d"], device="cuda")
        if own:
            _plan(s)
        return s
    s["seed"] = torch.randint(-2 ** 62, 2 ** 62, (2,), generator=g, device="cuda")
    if c["op"] == "drop":
        s["x"] = normal(c["M"], c["n"]).to(t)
        s["base"] = normal(c["M"], c["n"]).to(t) if c["base"] else None
        s["y"] = torch.empty_like(s["x"])
        return s
    M, K, N, r, n, lens = c["tokens"], c["K"], c["N"], c["rank"], c["adapters"], _lengths(c)
    s["lens"], s["ids"] = lens, _ids(c)                                              # a program knows them: it made the batch
    s["offsets"] = torch.tensor([sum(lens[:i]) for i in range(len(lens) + 1)], dtype=torch.int32, device="cuda")
    s["adapters"] = torch.tensor(s["ids"], dtype=torch.int32, device="cuda")
    s["scales"] = 0.5 + 1.5 * torch.rand(n, generator=g, device="cuda")
    s["a"] = [(normal(n, r, K) * K ** -0.5).to(t) for _ in range(c["mats"])]
    s["b"] = [(normal(n, N, r) * 0.1).to(t) for _ in range(c["mats"])]
    s["x"] = [normal(M, K).to(t) for _ in range(c["mats"])]
    if c["op"] == "adapter":
        yt = TYPES[c["y"]]
        s["base"] = [normal(M, N).to(yt) for _ in range(c["mats"])]                  # what the frozen projection gave
        s["y"] = [torch.empty(M, N, dtype=yt, device="cuda") for _ in range(c["mats"])]
        s["h"] = [torch.empty(M, r, device="cuda") for _ in range(c["mats"])] if c["p"] > 0.0 else None      # for the backward pass
    else:
        s["h"] = [h for _, h in _products(s)]                                        # as the forward pass left them
        s["dy"] = [normal(M, N).to(t) for _ in range(c["mats"])]
        s["base"] = [normal(M, K).to(t) for _ in range(c["mats"])]                   # gradient through the frozen projection
        s["dx"] = [torch.empty(M, K, dtype=t, device="cuda") for _ in range(c["mats"])]
        s["da"] = [torch.empty(n, r, K, device="cuda") for _ in range(c["mats"])]
        s["db"] = [torch.empty(n, N, r, device="cuda") for _ in range(c["mats"])]
    if own:
        _plan(s)
    return s


def _plan(s):
    """What a program keeps from call to call: descriptions of the rows and of the matrices, the workspace."""
    from paper_2505_03803_amd import binding as B
    c = s["case"]
    if c["op"] == "embed":
        return
    if c["op"] == "embed_grad":
        size = B.rwkvq_embedding_backward_workspace_size(c["tokens"], c["d"])
    else:
        alike = len(set(s["lens"])) == 1
        s["rows"] = B.AdapterRows(c["seqs"], c["tokens"], c["adapters"], c["rank"], offsets=None if alike else s["offsets"], adapters=s["adapters"],
                                  scales=s["scales"], seed=s["seed"] if c["p"] > 0.0 else None, p=c["p"])
        if c["op"] == "adapter":
            s["table"] = B.AdapterTable(s["a"], s["b"], s["x"], s["y"], bases=s["base"], hs=s["h"])
            return
        s["table"] = B.AdapterGradTable(s["a"], s["b"], s["x"], s["h"], s["dy"], s["dx"], s["da"], s["db"], bases=s["base"])
        size = B.rwkvq_adapters_backward_workspace_size(s["rows"], s["table"])
    s["workspace"] = torch.empty(max(size, 16), dtype=torch.uint8, device="cuda")


# ---- one pass ---------------------------------------------------------------------------------------------------

def run(s):
    return (_own if own else _plain)[s["case"]["op"]](s)


def _own_embed(s):
    from paper_2505_03803_amd import binding as B
    c = s["case"]
    B.rwkvq_embedding(s["tokens"], c["tokens"], s["table"], B.DTYPES[c["table"]], c["vocab"], c["d"], c["scale"], s["out"], B.DTYPES[c["x"]])
    return s["out"]


def _own_embed_grad(s):
    from paper_2505_03803_amd import binding as B
    c = s["case"]
    B.rwkvq_embedding_backward(s["tokens"], c["tokens"], s["dout"], B.DTYPES[c["x"]], c["vocab"], c["d"], c["scale"], s["dtable"], c["added"],
                               s["workspace"])
    return s["dtable"]


def _own_drop(s):
    from paper_2505_03803_amd import binding as B
    c = s["case"]
    B.rwkvq_dropout(s["x"], B.DTYPES[c["x"]], c["M"], c["n"], s["seed"], c["p"], s["y"], base=s["base"])
    return s["y"]


def _own_adapter(s):
    from paper_2505_03803_amd import binding as B
    c = s["case"]
    B.rwkvq_adapters(s["rows"], s["table"], B.DTYPES[c["x"]], B.DTYPES[c["y"]])
    return s["y"], s["h"]


def _own_adapter_grad(s):
    from paper_2505_03803_amd import binding as B
    B.rwkvq_adapters_backward(s["rows"], s["table"], B.DTYPES[s["case"]["x"]], s["workspace"])
    return s["dx"], s["da"], s["db"]


_own = {"embed": _own_embed, "embed_grad": _own_embed_grad, "drop": _own_drop, "adapter": _own_adapter, "adapter_grad": _own_adapter_grad}


# The plain forms: binary32 throughout, one rounding at the end.

def _plain_embed(s):
    live = s["tokens"] >= 0
    rows = s["table"][s["tokens"].clamp(min=0).long()].float() * s["case"]["scale"]
    return (rows * live[:, None]).to(s["out"].dtype)


def _plain_embed_grad(s):
    c = s["case"]
    live = s["tokens"] >= 0
    sums = torch.zeros(c["vocab"], c["d"], device="cuda").index_add_(0, s["tokens"].clamp(min=0).long(), s["dout"].float() * live[:, None])
    if not c["added"]:
        return sums * c["scale"]
    s["dtable"] += sums * c["scale"]
    return s["dtable"]


def _keep(seed, call, M, n, p):
    """[M][n]: which elements stay, and the factor of those that do.  Products of 32-bit words are taken in int64, whose wrapped bits are right."""
    limit = int(p * 65536.0 + 0.5)
    low = 0xFFFFFFFF
    blocks = (n + 7) // 8
    c0 = torch.arange(blocks, device="cuda").expand(M, blocks)
    c1 = torch.arange(M, device="cuda")[:, None].expand(M, blocks)
    number = seed[1] + call
    c2, c3 = (number & low).expand(M, blocks), (number >> 32 & low).expand(M, blocks)
    k0, k1 = seed[0] & low, seed[0] >> 32 & low
    for _ in range(10):
        a, b = c0 * 0xD2511F53, c2 * 0xCD9E8D57
        c0, c1, c2, c3 = (b >> 32 & low) ^ c1 ^ k0, b & low, (a >> 32 & low) ^ c3 ^ k1, a & low
        k0, k1 = k0 + 0x9E3779B9 & low, k1 + 0xBB67AE85 & low
    words = torch.stack([c0, c1, c2, c3], -1)
    numbers = torch.stack([words & 0xFFFF, words >> 16], -1).reshape(M, -1)[:, :n]
    return numbers >= limit, 65536.0 / (65536.0 - limit)


def _dropped(s, x, call=0):
    c = s["case"]
    if c["p"] == 0.0:
        return x
    keep, factor = _keep(s["seed"], call, x.shape[0], x.shape[1], c["p"])
    return torch.where(keep, x * factor, 0.0)


def _plain_drop(s):
    y = _dropped(s, s["x"].float())
    return (y if s["base"] is None else s["base"].float() + y).to(s["x"].dtype)


def _runs(s):
    """(adapter, rows) of each sequence; single tokens of all sequences at once."""
    c = s["case"]
    first = [sum(s["lens"][:i]) for i in range(c["seqs"])]
    return [(a, slice(f, f + n)) for a, f, n in zip(s["ids"], first, s["lens"]) if n and a >= 0]


def _products(s):
    """For each matrix what is added to the projection, and h."""
    c = s["case"]
    single = max(s["lens"]) == 1 and len(s["lens"]) == c["tokens"]
    for i in range(c["mats"]):
        x = _dropped(s, s["x"][i].float(), i)
        h = torch.zeros(c["tokens"], c["rank"], device="cuda")
        z = torch.zeros(c["tokens"], c["N"], device="cuda")
        if single:
            ids, live = s["adapters"].clamp(min=0).long(), (s["adapters"] >= 0)[:, None]
            h = (s["a"][i][ids].float() @ x[..., None])[..., 0] * live
            z = (s["b"][i][ids].float() @ h[..., None])[..., 0] * s["scales"][ids][:, None]
        else:
            for a, rows in _runs(s):
                h[rows] = x[rows] @ s["a"][i][a].float().T
                z[rows] = h[rows] @ s["b"][i][a].float().T * s["scales"][a]
        yield z, h


def _plain_adapter(s):
    ys, hs = [], []
    for base, (z, h) in zip(s["base"], _products(s)):
        ys.append((base.float() + z).to(base.dtype))
        hs.append(h)
    return ys, hs if s["h"] is not None else None


def _plain_adapter_grad(s):
    c = s["case"]
    dxs, das, dbs = [], [], []
    for i in range(c["mats"]):
        x, dy = _dropped(s, s["x"][i].float(), i), s["dy"][i].float()
        back = torch.zeros(c["tokens"], c["K"], device="cuda")
        da, db = torch.zeros_like(s["da"][i]), torch.zeros_like(s["db"][i])
        for a, rows in _runs(s):
            g = dy[rows] @ s["b"][i][a].float() * s["scales"][a]
            back[rows] = g @ s["a"][i][a].float()
            da[a] += g.T @ x[rows]
            db[a] += dy[rows].T @ s["h"][i][rows] * s["scales"][a]
        dxs.append((s["base"][i].float() + _dropped(s, back, i)).to(s["dx"][i].dtype))
        das.append(da)
        dbs.append(db)
    return dxs, das, dbs


_plain = {"embed": _plain_embed, "embed_grad": _plain_embed_grad, "drop": _plain_drop, "adapter": _plain_adapter, "adapter_grad": _plain_adapter_grad}


# ---- what a pass cannot do without ------------------------------------------------------------------------------

def work(c):
    size = {"f16": 2, "bf16": 2, "f32": 4}
    x = size[c["x"]]
    if c["op"] == "drop":
        # ten rounds of two products and four more operations on words of 32 bits for eight elements
        return {"bytes": (3 if c["base"] else 2) * c["M"] * c["n"] * x, "flops": 10 * c["M"] * c["n"]}
    if c["op"].startswith("embed"):
        tokens = _tokens(c)
        live, rows = int((tokens >= 0).sum()), len(set(tokens[tokens >= 0].tolist()))
        if c["op"] == "embed":
            return {"bytes": (rows * size[c["table"]] + c["tokens"] * x) * c["d"] + 4 * c["tokens"], "flops": c["tokens"] * c["d"]}
        return {"bytes": (live * x + (8 * rows if c["added"] else 4 * c["vocab"])) * c["d"] + 4 * c["tokens"], "flops": 2 * live * c["d"]}
    M, K, N, r = c["tokens"], c["K"], c["N"], c["rank"]
    lens, ids = _lengths(c), _ids(c)
    used = len({a for a, n in zip(ids, lens) if n and a >= 0})
    live = sum(n for a, n in zip(ids, lens) if a >= 0)
    weights = used * r * (K + N) * x
    if c["op"] == "adapter":
        return {"bytes": c["mats"] * (live * K * x + 2 * M * N * size[c["y"]] + weights + (4 * M * r if c["p"] > 0.0 else 0)),
                "flops": c["mats"] * 2 * live * r * (K + N)}
    return {"bytes": c["mats"] * (live * (K + N) * x + 2 * M * K * x + weights + 4 * live * r + 4 * c["adapters"] * r * (K + N)),
            "flops": c["mats"] * 4 * live * r * (K + N)}


# ---- the definition in 64 bits ----------------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    return {"embed": _exact_embed, "embed_grad": _exact_embed_grad, "drop": _exact_drop, "adapter": _exact_adapter,
            "adapter_grad": _exact_adapter_grad}[case["op"]](s)


def _exact_embed(s):
    table = torch.cat([s["table"], torch.zeros_like(s["table"][:1])])                # padding, -1, is the row behind the last
    return table[s["tokens"].long()].double() * s["case"]["scale"]


def _exact_embed_grad(s):
    c = s["case"]
    out = s["dtable"].double() if c["added"] else torch.zeros(c["vocab"], c["d"], dtype=torch.float64, device="cuda")
    rows = s["dout"].double() * c["scale"]
    tokens = s["tokens"].tolist()
    order = sorted(range(c["tokens"]), key=tokens.__getitem__)
    values = [tokens[i] for i in order]
    places = torch.tensor(order, device="cuda")
    at = 0
    while at < len(values):
        end = at + 1
        while end < len(values) and values[end] == values[at]:
            end += 1
        if values[at] >= 0:
            out[values[at]] += rows[places[at:end]].sum(0)
        at = end
    return out


def _numbers(key, call, M, blocks):
    """The generator with numpy's unsigned words: [M][8 blocks] numbers of 16 bits."""
    u = np.uint64
    low, half = u(0xFFFFFFFF), u(32)
    x = [np.broadcast_to(np.arange(blocks, dtype=u), (M, blocks)), np.broadcast_to(np.arange(M, dtype=u)[:, None], (M, blocks)),
         np.full((M, blocks), u(call & 0xFFFFFFFF)), np.full((M, blocks), u(call >> 32))]
    k = [key & 0xFFFFFFFF, key >> 32]
    for _ in range(10):
        p, q = x[0] * u(0xD2511F53), x[2] * u(0xCD9E8D57)
        x = [(q >> half) ^ x[1] ^ u(k[0]), q & low, (p >> half) ^ x[3] ^ u(k[1]), p & low]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    out = np.empty((M, blocks, 8), dtype=np.uint16)
    for w in range(4):
        out[..., 2 * w] = (x[w] & u(0xFFFF)).astype(np.uint16)
        out[..., 2 * w + 1] = (x[w] >> u(16)).astype(np.uint16)
    return out.reshape(M, -1)


def _factors(s, M, n, call=0):
    """0 or 1 / (1 - p) for each element, p as a multiple of 2^-16."""
    p = s["case"]["p"]
    if p == 0.0:
        return 1.0
    key, number = (v % 2 ** 64 for v in s["seed"].tolist())
    limit = math.floor(p * 65536.0 + 0.5)
    keep = _numbers(key, (number + call) % 2 ** 64, M, -(-n // 8))[:, :n] >= limit
    return torch.from_numpy(keep).cuda().double() / (1.0 - limit / 65536.0)


def _exact_drop(s):
    y = s["x"].double() * _factors(s, *s["x"].shape)
    return y if s["base"] is None else y + s["base"].double()


def _exact_rows(s):
    """The adapter of each row, -1 where it has none."""
    return torch.tensor([a for a, n in zip(s["ids"], s["lens"]) for _ in range(n)], device="cuda")


def _exact_adapter(s):
    c = s["case"]
    row = _exact_rows(s)
    ys, hs = [], []
    for i in range(c["mats"]):
        x = s["x"][i].double() * _factors(s, c["tokens"], c["K"], i)
        y, h = s["base"][i].double(), torch.zeros(c["tokens"], c["rank"], dtype=torch.float64, device="cuda")
        for a in range(c["adapters"]):
            at = torch.nonzero(row == a)[:, 0]
            if len(at):
                h[at] = torch.mm(s["a"][i][a].double(), x[at].T).T
                y[at] += s["scales"][a].double() * torch.mm(s["b"][i][a].double(), h[at].T).T
        ys.append(y)
        hs.append(h)
    return ys, hs if s["h"] is not None else None


def _exact_adapter_grad(s):
    c = s["case"]
    row = _exact_rows(s)
    dxs, das, dbs = [], [], []
    for i in range(c["mats"]):
        factor = _factors(s, c["tokens"], c["K"], i)
        x, dx = s["x"][i].double() * factor, torch.zeros(c["tokens"], c["K"], dtype=torch.float64, device="cuda")
        da, db = (torch.zeros_like(t, dtype=torch.float64) for t in (s["da"][i], s["db"][i]))
        for a in range(c["adapters"]):
            at = torch.nonzero(row == a)[:, 0]
            if len(at):
                A, Bm = s["a"][i][a].double(), s["scales"][a].double() * s["b"][i][a].double()
                g = torch.mm(s["dy"][i][at].double(), Bm)
                dx[at] = torch.mm(g, A)
                da[a] = torch.mm(g.T, x[at])
                db[a] = s["scales"][a].double() * torch.mm(s["dy"][i][at].double().T, s["h"][i][at].double())
        dxs.append(s["base"][i].double() + dx * factor)
        das.append(da)
        dbs.append(db)
    return dxs, das, dbs
