"""A multi-head time-mixing block over frozen quantized projections, written with the library's entry points: prompts of several
sequences at once, one token of each (also as a HIP graph), and the gradients of what is tuned around the frozen matrices.

    a    = norm(x; ln)                                      rwkvq_layer_norm, whole rows
    x_p  = mu_p a_t + (1 - mu_p) a_{t-1},  p in r, k, v, g  rwkvq_token_shift_mix
    r, k, v, g = Deq(W_p) x_p                               rwkvq_linear_dispatch
    o    = attention(r, k, v; w, u)                         rwkvq_linear_attention, states in a pool, one slot a sequence
    z    = norm(o; heads)                                   rwkvq_layer_norm, a group for each head
    out  = Deq(W_o) (sigma(g) z)                            rwkvq_sigmoid_gate, rwkvq_linear_dispatch

Beside the five matrices there may be a pool of low-rank adapters (Adapters), of which a plan gives one to each sequence, or none:

    r, k, v, g += s_a B_ap (A_ap drop(x_p)),  out += s_a B_ao (A_ao drop(sigma(g) z))       rwkvq_adapters

python -m paper_2505_03803_amd.time_mix [--d 4096] [--heads 64] [--tokens 2048] [--steps 64] runs it on synthetic weights."""
from __future__ import annotations

import argparse
import time
from typing import Callable, Dict, Optional, Sequence, Tuple

import numpy as np
import torch

from . import binding as B
from . import synth

PROJECTIONS = ("r", "k", "v", "g")
TYPES = {B.F16: torch.float16, B.BF16: torch.bfloat16}


class Adapters:
    """A pool of n low-rank adapters for each projection of a block of width d: a [n][rank][d] and b [n][d][rank] of the block's type by
    projection, scales float32 [n].  p: dropout in front of them, in plans that ask for it; `seeds` holds the key and the number of the
    next call of the first four and of the last one, and advance() moves both on to other masks, also in a captured graph."""

    def __init__(self, d: int, n: int, rank: int, dtype: int = B.F16, p: float = 0.0, seed: int = 0, device: str = "cuda:0"):
        self.n, self.rank, self.p = n, rank, p
        gen = torch.Generator().manual_seed(seed)
        kind = TYPES[dtype]
        # as adapters begin: A random, B zero, so that a block without training is the block
        self.a = {q: (torch.randn(n, rank, d, generator=gen) * d ** -0.5).to(kind).to(device) for q in PROJECTIONS + ("o",)}
        self.b = {q: torch.zeros(n, d, rank, dtype=kind, device=device) for q in PROJECTIONS + ("o",)}
        self.scales = torch.ones(n, device=device)
        self.seeds = torch.tensor([[seed, 0], [seed, len(PROJECTIONS)]], dtype=torch.int64, device=device)

    def advance(self) -> None:
        self.seeds[:, 1] += len(PROJECTIONS) + 1


class TimeMix:
    """mats: the quantized matrices r, k, v, g, o (synth.QMatrix, d x d); mus: (indices uint8 [d / 2], codebook uint16 [2^kbits][2])
    of each of r, k, v, g; w: float32 [heads], u: float32 [heads][d / heads]; ln, heads_norm: (weight, bias), float32 [d].
    max_tokens bounds the rows of a call, n_slots is the size of the pool of states."""
    adapters: Optional[Adapters] = None

    def __init__(self, d: int, n_heads: int, mats: Dict[str, synth.QMatrix], mus: Dict[str, Tuple[np.ndarray, np.ndarray]], w, u, ln,
                 heads_norm, n_slots: int, max_tokens: int, kbits: int = 6, dtype: int = B.F16, eps: float = 1e-5,
                 device: str = "cuda:0", adapters: Optional[Adapters] = None):
        if adapters is not None:
            for p in PROJECTIONS + ("o",):
                a, b = adapters.a[p], adapters.b[p]
                if a.dtype != TYPES[dtype] or b.dtype != TYPES[dtype] or a.shape != (adapters.n, adapters.rank, d) or b.shape != (adapters.n, d, adapters.rank):
                    raise ValueError(f"adapters {tuple(a.shape)}, {tuple(b.shape)} of {a.dtype} in a block of width {d} of {TYPES[dtype]}")
        self.d, self.H, self.D, self.dtype, self.eps, self.kbits = d, n_heads, d // n_heads, dtype, eps, kbits
        self.device, self.n_slots, self.max_tokens = device, n_slots, max_tokens
        self.mats = {p: B.upload(mats[p], device=device) for p in PROJECTIONS + ("o",)}
        self.indices = [torch.from_numpy(np.ascontiguousarray(mus[p][0])).to(device) for p in PROJECTIONS]
        self.codebooks = [torch.from_numpy(np.ascontiguousarray(mus[p][1]).view(np.int16)).to(device) for p in PROJECTIONS]
        f32 = lambda a: torch.as_tensor(a, dtype=torch.float32).contiguous().to(device)
        self.w, self.u = f32(w), f32(u)
        self.ln, self.heads_norm = tuple(map(f32, ln)), tuple(map(f32, heads_norm))
        self.state = torch.zeros(n_slots, self.H, self.D, self.D, device=device)
        self.last = torch.zeros(n_slots, d, dtype=TYPES[dtype], device=device)       # a of each sequence's last token
        rows = lambda n: torch.empty(n, max_tokens, d, dtype=TYPES[dtype], device=device)
        self.a, self.o, self.z, self.gated, self.out = rows(5)
        self.mixed, self.proj = rows(4), rows(4)
        self.stats = [torch.empty(max_tokens, n, device=device) for n in (1, 1, self.H, self.H)]
        if adapters is not None:
            self.adapters = adapters
            self.seeds = torch.zeros_like(adapters.seeds)           # those of the masks of the call whose rows the buffers hold
            self.h = {p: torch.empty(max_tokens, adapters.rank, device=device) for p in PROJECTIONS + ("o",)}
        self.dense: Optional[Dict[str, torch.Tensor]] = None
        self.holds = None, None                                     # x and plan of the call whose rows the buffers hold

    def _heads(self, lens: Sequence[int], slots: Optional[Sequence[int]]) -> B.Heads:
        i32 = lambda a: torch.tensor(a, dtype=torch.int32, device=self.device)
        offsets = None if len(set(lens)) == 1 else i32(np.concatenate([[0], np.cumsum(lens)]))
        return B.Heads(len(lens), sum(lens), self.H, self.D, offsets, None if slots is None else i32(list(slots)),
                       0 if slots is None else self.n_slots)

    def _rows(self, lens: Sequence[int], ids: Sequence[int], drop: bool):
        """The descriptions of the rows for the adapters of the first four projections and of the last."""
        i32 = lambda a: torch.tensor(a, dtype=torch.int32, device=self.device)
        offsets = None if len(set(lens)) == 1 else i32(np.concatenate([[0], np.cumsum(lens)]))
        pool = self.adapters
        return [B.AdapterRows(len(lens), sum(lens), pool.n, pool.rank, offsets, i32(list(ids)), pool.scales, seed if drop and pool.p > 0 else None, pool.p)
                for seed in pool.seeds]

    def plan(self, lens: Sequence[int], slots: Optional[Sequence[int]] = None, adapters: Optional[Sequence[int]] = None, drop: bool = False):
        """What calls of one form share: the sequences' lengths, their slots (None: they begin empty and leave no state), and the
        workspace.  A captured graph replays one plan.  Each sequence has a slot of the pool to itself.  adapters: that of each sequence, -1
        for none (None: the block without adapters); drop: with dropout in front of them.  -> lens, slots, heads, workspace, and of a block with
        adapters their rows, or None"""
        if min(lens) < 0 or sum(lens) > self.max_tokens:
            raise ValueError(f"sequences of {list(lens)} tokens in a block for at most {self.max_tokens}")
        if slots is not None and (len(slots) != len(lens) or len(set(slots)) != len(lens) or not all(0 <= s < self.n_slots for s in slots)):
            raise ValueError(f"slots {list(slots)} for {len(lens)} sequences in a pool of {self.n_slots}")
        if adapters is not None and (self.adapters is None or len(adapters) != len(lens) or not all(-1 <= a < self.adapters.n for a in adapters)):
            raise ValueError(f"adapters {list(adapters)} for {len(lens)} sequences in a block with {self.adapters.n if self.adapters else 0}")
        heads = self._heads(lens, slots)
        n = B.rwkvq_linear_attention_workspace_size(heads)
        plan = lens, slots, heads, torch.empty(max(n, 16), dtype=torch.uint8, device=self.device)
        return plan if self.adapters is None else (*plan, None if adapters is None else self._rows(lens, adapters, drop))

    def _adapt(self, rows: B.AdapterRows, projections: Sequence[str], xs, ys) -> None:
        pool = self.adapters
        table = B.AdapterTable([pool.a[p] for p in projections], [pool.b[p] for p in projections], xs, ys, bases=ys, hs=[self.h[p] for p in projections])
        B.rwkvq_adapters(rows, table, self.dtype, self.dtype)

    def _adapt_backward(self, rows: B.AdapterRows, projections: Sequence[str], xs, dys, dxs):
        """Adds the adapters' share to dxs.  -> (da, db) by projection"""
        pool = self.adapters
        grads = {p: (torch.empty(pool.a[p].shape, device=self.device), torch.empty(pool.b[p].shape, device=self.device)) for p in projections}
        table = B.AdapterGradTable([pool.a[p] for p in projections], [pool.b[p] for p in projections], xs, [self.h[p] for p in projections], dys, dxs,
                                   [grads[p][0] for p in projections], [grads[p][1] for p in projections], bases=dxs)
        workspace = torch.empty(B.rwkvq_adapters_backward_workspace_size(rows, table), dtype=torch.uint8, device=self.device)
        B.rwkvq_adapters_backward(rows, table, self.dtype, workspace)
        return grads

    def forward(self, x: torch.Tensor, plan) -> torch.Tensor:
        """x: [tokens][d], the sequences' rows one after the other.  -> [tokens][d], a view that the next call overwrites"""
        lens, slots, heads, workspace, rows = plan if len(plan) == 5 else (*plan, None)
        T, H, dt = sum(lens), self.H, self.dtype
        self.holds = x, plan
        if rows and rows[0].seed is not None:
            for kept, r in zip(self.seeds, rows):
                kept.copy_(r.seed)
        mean, rstd, head_mean, head_rstd = self.stats
        B.rwkvq_layer_norm(x, dt, T, 1, self.d, *self.ln, self.eps, self.a, mean, rstd)
        first = 0
        for i, n in enumerate(lens):
            if n:
                last = self.last[slots[i]] if slots is not None else torch.zeros_like(self.last[0])
                table = B.MixTable(self.indices, self.codebooks, [m[first:] for m in self.mixed])
                B.rwkvq_token_shift_mix(self.a[first:], last, dt, n, self.d, table, self.kbits)
                if slots is not None:
                    last.copy_(self.a[first + n - 1])
            first += n
        B.rwkvq_linear_dispatch(B.DispatchTable([self.mats[p].desc() for p in PROJECTIONS], list(self.mixed), list(self.proj)), T, dt, dt)
        if rows:
            self._adapt(rows[0], PROJECTIONS, list(self.mixed), list(self.proj))
        r, k, v, g = self.proj
        state = None if slots is None else self.state
        B.rwkvq_linear_attention(heads, r, k, v, dt, self.w, self.u, state, state, self.o, workspace)
        B.rwkvq_layer_norm(self.o, dt, T, H, self.D, *self.heads_norm, self.eps, self.z, head_mean, head_rstd)
        B.rwkvq_sigmoid_gate(g, self.z, dt, T * self.d, self.gated)
        B.rwkvq_linear_dispatch(B.DispatchTable([self.mats["o"].desc()], [self.gated], [self.out]), T, dt, dt)
        if rows:
            self._adapt(rows[1], ("o",), [self.gated], [self.out])
        return self.out[:T]

    def capture(self, x: torch.Tensor, plan) -> Callable[[], torch.Tensor]:
        """forward(x, plan) as a HIP graph: write the next tokens into x and call what is returned.  Capturing leaves the states as
        they are."""
        keep = self.state.clone(), self.last.clone()
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            self.forward(x, plan)
        torch.cuda.current_stream().wait_stream(side)
        self.state.copy_(keep[0]); self.last.copy_(keep[1])
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = self.forward(x, plan)

        def replay(keep=(self, x, plan)):                            # the graph reads and writes the buffers of all three
            self.holds = x, plan
            graph.replay()
            return out

        return replay

    def backward(self, x: torch.Tensor, dout: torch.Tensor, plan) -> Dict[str, torch.Tensor]:
        """The gradients behind forward(x, plan), the last call before this one, with a plan without slots: of x, both norms, w, u and, where
        the plan has them, the adapters, with the masks that the call had, whatever the pool's seeds are by now.  The products with the
        transposed matrices are taken on their dense copies, made at the first call."""
        lens, slots, heads, _, rows = plan if len(plan) == 5 else (*plan, None)
        if slots is not None:
            raise ValueError("gradients of sequences that begin with a state of the pool")
        if self.holds[1] is not plan or self.holds[0].data_ptr() != x.data_ptr():        # x itself or a view of its rows
            raise ValueError("gradients of a call whose rows the block does not hold any more")
        if rows and rows[0].seed is not None:
            rows = [r.with_seed(kept) for r, kept in zip(rows, self.seeds)]
        T, H, D, d, dt = sum(lens), self.H, self.D, self.d, self.dtype
        kind = TYPES[dt]
        if self.dense is None:
            self.dense = {p: B.dequant(m, dt).view(kind) for p, m in self.mats.items()}
        mean, rstd, head_mean, head_rstd = self.stats
        r, k, v, g = (p[:T] for p in self.proj)
        like = lambda: torch.empty(T, d, dtype=kind, device=self.device)
        f32 = lambda *shape: torch.empty(shape, device=self.device)
        scratch = lambda n: torch.empty(max(n, 16), dtype=torch.uint8, device=self.device)

        dgated = dout @ self.dense["o"]
        tuned = self._adapt_backward(rows[1], ("o",), [self.gated], [dout.contiguous()], [dgated]) if rows else {}
        dgated = dgated.float()
        s = torch.sigmoid(g.float())
        dz, dg = (dgated * s).to(kind), (dgated * self.z[:T].float() * s * (1 - s)).to(kind)
        do, dheads_w, dheads_b = like(), f32(d), f32(d)
        B.rwkvq_layer_norm_backward(dz, self.o, dt, T, H, D, self.heads_norm[0], head_mean, head_rstd, do, dheads_w, dheads_b,
                                    scratch(B.rwkvq_layer_norm_backward_workspace_size(T, H, D)))
        dr, dk, dv, dw, du = like(), like(), like(), f32(H), f32(H, D)
        B.rwkvq_linear_attention_backward(heads, r, k, v, do, dt, self.w, self.u, None, None, dr, dk, dv, dw, du, None,
                                          scratch(B.rwkvq_linear_attention_backward_workspace_size(heads)))
        da = torch.zeros(T, d, device=self.device)
        starts = np.concatenate([[0], np.cumsum(lens)])
        inner = torch.ones(T, 1, device=self.device)                # 0 at the first token of a sequence: nothing is in front of it
        inner[[int(f) for f, n in zip(starts, lens) if n]] = 0
        through = [grad @ self.dense[p] for p, grad in zip(PROJECTIONS, (dr, dk, dv, dg))]
        if rows:
            tuned.update(self._adapt_backward(rows[0], PROJECTIONS, list(self.mixed), [dr, dk, dv, dg], through))
        for dx, index, book in zip(through, self.indices, self.codebooks):
            mu = book.view(torch.float16).view(-1, 2)[index.long()].reshape(-1).float()
            dx = dx.float()
            da += mu * dx
            da[:-1] += ((1 - mu) * dx * inner)[1:]
        dx, dln_w, dln_b = like(), f32(d), f32(d)
        B.rwkvq_layer_norm_backward(da.to(kind), x, dt, T, 1, d, self.ln[0], mean, rstd, dx, dln_w, dln_b,
                                    scratch(B.rwkvq_layer_norm_backward_workspace_size(T, 1, d)))
        grads = dict(x=dx, ln=(dln_w, dln_b), heads_norm=(dheads_w, dheads_b), w=dw, u=du)
        return dict(grads, adapters=tuned) if rows else grads


def synthetic(d: int, n_heads: int, n_slots: int, max_tokens: int, seed: int = 0, dtype: int = B.F16,
              adapters: Optional[Adapters] = None) -> TimeMix:
    """A block with random weights of the shapes and spreads of the repository's other synthetic workloads."""
    rng = np.random.default_rng(seed)
    mats = {p: synth.gen_sq(rng, d, d, p) if i % 2 else synth.gen_vq(rng, d, d, 6, p) for i, p in enumerate(PROJECTIONS + ("o",))}
    mus = {p: (rng.integers(0, 64, size=d // 2, dtype=np.uint8), synth.gen_codebook(rng, 64)) for p in PROJECTIONS}
    w = np.exp(rng.uniform(-5.0, 1.0, size=n_heads))
    u = 0.5 * rng.standard_normal((n_heads, d // n_heads))
    norms = [(1 + 0.1 * rng.standard_normal(d), 0.1 * rng.standard_normal(d)) for _ in range(2)]
    return TimeMix(d, n_heads, mats, mus, w, u, norms[0], norms[1], n_slots, max_tokens, dtype=dtype, adapters=adapters)


def timed(f: Callable[[], object], n: int) -> float:
    """Seconds of a call, behind one that is not counted."""
    f()
    torch.cuda.synchronize()
    t = time.perf_counter()
    for _ in range(n):
        f()
    torch.cuda.synchronize()
    return (time.perf_counter() - t) / n


def main() -> None:
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--d", type=int, default=4096)
    ap.add_argument("--heads", type=int, default=64)
    ap.add_argument("--tokens", type=int, default=2048, help="tokens of the prompt and of the training step")
    ap.add_argument("--steps", type=int, default=64, help="single tokens behind the prompt")
    args = ap.parse_args()
    block = synthetic(args.d, args.heads, 1, args.tokens)
    x = torch.randn(args.tokens, args.d, device="cuda").to(TYPES[block.dtype])

    prompt = block.plan([args.tokens], [0])
    t = timed(lambda: block.forward(x, prompt), 5)
    print(f"prompt of {args.tokens} tokens: {t * 1e3:.3f} ms, {args.tokens / t:.0f} tokens/s")
    token = x[:1].clone()
    t = timed(block.capture(token, block.plan([1], [0])), args.steps)
    print(f"one token as a HIP graph: {t * 1e6:.1f} us")
    train = block.plan([args.tokens])

    def step():
        y = block.forward(x, train)
        block.backward(x, y.clone(), train)

    t = timed(step, 5)
    print(f"forward and backward of {args.tokens} tokens: {t * 1e3:.3f} ms")


if __name__ == "__main__":
    main()
