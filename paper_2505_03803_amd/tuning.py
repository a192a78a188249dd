"""A step of tuning around a frozen quantized block: the rows of a table by token, the block with low-rank adapters beside its matrices,
dropout and a residual, and the gradients of the table, the adapters and the block's own vectors.

    x   = table[token]                                      rwkvq_embedding
    out = x + drop(block(x))                                time_mix.TimeMix with Adapters, rwkvq_dropout
    dtable_v = sum of dx over the tokens v                  rwkvq_embedding_backward

python -m paper_2505_03803_amd.tuning [--d 4096] [--heads 64] [--tokens 2048] [--rank 16] [--vocab 65536] runs it on synthetic weights."""
from __future__ import annotations

import argparse
from typing import Dict, Optional, Sequence

import torch

from . import binding as B
from . import time_mix


class Tuning:
    """table: [vocab][d] of the block's type.  p: dropout of the block's output; `seed` holds its key and the number of the next call; a key
    other than the adapters', whose numbers begin at 0 as well."""

    def __init__(self, block: time_mix.TimeMix, table: torch.Tensor, p: float = 0.0, seed: int = 1):
        if table.dtype != time_mix.TYPES[block.dtype] or table.dim() != 2 or table.shape[1] != block.d or not table.is_contiguous():
            raise ValueError(f"a table {tuple(table.shape)} of {table.dtype} for a block of width {block.d} of {time_mix.TYPES[block.dtype]}")
        self.block, self.table, self.p = block, table, p
        self.vocab, self.d = table.shape
        self.seed = torch.tensor([seed, 0], dtype=torch.int64, device=table.device)
        self.drawn, self.drawn_p = torch.zeros_like(self.seed), p           # those of the call before
        rows = lambda: torch.empty(block.max_tokens, self.d, dtype=table.dtype, device=table.device)
        self.x, self.out, self.dy = rows(), rows(), rows()
        self.holds: Optional[torch.Tensor] = None                           # tokens of the call whose rows x holds

    def plan(self, lens: Sequence[int], adapters: Optional[Sequence[int]] = None):
        """Sequences that begin empty, and the adapter of each."""
        return self.block.plan(lens, adapters=adapters, drop=True)

    def _count(self, tokens: torch.Tensor, plan) -> int:
        T = sum(plan[0])
        if tokens.dtype != torch.int32 or tokens.shape != (T,) or not tokens.is_contiguous():
            raise ValueError(f"{tuple(tokens.shape)} tokens of {tokens.dtype} for a plan of {T}, which takes int32 one after the other")
        return T

    def forward(self, tokens: torch.Tensor, plan) -> torch.Tensor:
        """tokens: int32, the sequences' one after the other; one outside the table is padding, a row of zeros.  -> [tokens][d], a view that the next
        call overwrites"""
        T, dt = self._count(tokens, plan), self.block.dtype
        self.holds = tokens
        B.rwkvq_embedding(tokens, T, self.table, dt, self.vocab, self.d, 1.0, self.x, dt)
        y = self.block.forward(self.x[:T], plan)
        self.drawn_p = self.p
        self.drawn.copy_(self.seed)
        B.rwkvq_dropout(y, dt, T, self.d, self.drawn, self.drawn_p, self.out, base=self.x)
        return self.out[:T]

    def backward(self, tokens: torch.Tensor, dout: torch.Tensor, plan, dtable: torch.Tensor, accumulate: bool = False) -> Dict[str, object]:
        """The gradients behind forward(tokens, plan), the last call before this one, with the masks that it had, also after advance(): those of the
        block, and dtable (float32 [vocab][d], overwritten or added to).  tokens: the tensor that this call had."""
        T, dt = self._count(tokens, plan), self.block.dtype
        if dout.shape != (T, self.d) or dout.dtype != self.table.dtype:
            raise ValueError(f"a gradient {tuple(dout.shape)} of {dout.dtype} for {T} tokens")
        if dtable.shape != self.table.shape or dtable.dtype != torch.float32 or not dtable.is_contiguous():
            raise ValueError(f"a table's gradient {tuple(dtable.shape)} of {dtable.dtype}")
        if self.holds is None or self.holds.data_ptr() != tokens.data_ptr():
            raise ValueError("gradients of tokens whose rows the step does not hold any more")
        dout = dout.contiguous()
        B.rwkvq_dropout(dout, dt, T, self.d, self.drawn, self.drawn_p, self.dy)
        grads = self.block.backward(self.x[:T], self.dy[:T], plan)
        dx = grads.pop("x").float() + dout                        # binary32: the table's gradient is a sum of these
        workspace = torch.empty(B.rwkvq_embedding_backward_workspace_size(T, self.d), dtype=torch.uint8, device=self.table.device)
        B.rwkvq_embedding_backward(tokens, T, dx, B.F32, self.vocab, self.d, 1.0, dtable, accumulate, workspace)
        return dict(grads, table=dtable)

    def advance(self) -> None:
        """Other masks for the next step."""
        self.seed[1] += 1
        if self.block.adapters is not None:
            self.block.adapters.advance()


def main() -> None:
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--d", type=int, default=4096)
    ap.add_argument("--heads", type=int, default=64)
    ap.add_argument("--tokens", type=int, default=2048)
    ap.add_argument("--rank", type=int, default=16)
    ap.add_argument("--vocab", type=int, default=65536)
    args = ap.parse_args()
    pool = time_mix.Adapters(args.d, 1, args.rank, p=0.05)
    block = time_mix.synthetic(args.d, args.heads, 1, args.tokens, adapters=pool)
    step = Tuning(block, (0.02 * torch.randn(args.vocab, args.d, device="cuda")).half(), p=0.1)
    tokens = torch.randint(0, args.vocab, (args.tokens,), device="cuda").to(torch.int32)
    dtable = torch.empty(args.vocab, args.d, device="cuda")

    def timed(plan):
        def one():
            out = step.forward(tokens, plan)
            step.backward(tokens, out.clone(), plan, dtable)
            step.advance()
        return time_mix.timed(one, 5)

    bare, tuned = timed(step.plan([args.tokens])), timed(step.plan([args.tokens], [0]))
    print(f"forward and backward of {args.tokens} tokens: {tuned * 1e3:.3f} ms, without adapters {bare * 1e3:.3f} ms")


if __name__ == "__main__":
    main()
