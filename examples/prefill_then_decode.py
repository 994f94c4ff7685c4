"""Document pages from their first token to a branch-decode step.

The vision and prompt tokens of a few pages are prefilled in chunks into one
paged cache: every step takes pages of the pool for its new tokens (ChunkSlots),
and every layer normalises, rotates and caches its projection's rows (QkNormRope)
and attends to what the cache holds (ChunkAttn).  Content branches forked from the
pages then decode one step (BranchAttn), their shared prefix read where the
prefill left it.  Weights and inputs are random.

    python examples/prefill_then_decode.py
"""
import os
import sys
from dataclasses import dataclass

import numpy as np

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2607_18839_gb300 import hpd  # noqa: E402

PAGE = 16


@dataclass
class Shape:
    layers: int = 2
    hidden: int = 256
    H_q: int = 16
    H_kv: int = 2
    D: int = 128
    # frequencies turned by the place in time, by the row and by the column
    sections: tuple = (16, 24, 24)


class Pages:
    """A model's caches and the pages of some documents in them.

    grids: (rows, columns) of vision tokens of each document, prompts: the text
    tokens behind them; room: tokens a step may bring; extra: pages left over."""

    def __init__(self, shape, grids, prompts, room, extra=64, seed=0, device="cuda"):
        import torch
        s, self.shape, self.room = shape, shape, room
        self.vision = [r * c for r, c in grids]
        self.total = [v + p for v, p in zip(self.vision, prompts)]
        S, held = len(grids), [-(-n // PAGE) for n in self.total]
        num_pages = sum(held) + extra
        gen = torch.Generator(device=device).manual_seed(seed)
        rand = lambda *n, std=1.0: (torch.randn(n, generator=gen, device=device) * std).bfloat16()  # noqa: E731
        i32 = dict(dtype=torch.int32, device=device)
        width = (s.H_q + 2 * s.H_kv) * s.D
        self.w_in = [rand(s.hidden, width, std=s.hidden ** -0.5) for _ in range(s.layers)]
        self.w_out = [rand(s.H_q * s.D, s.hidden, std=(s.H_q * s.D) ** -0.5) for _ in range(s.layers)]
        self.cache = [(torch.zeros(num_pages, PAGE, s.H_kv, s.D, dtype=torch.bfloat16, device=device),
                       torch.zeros(num_pages, PAGE, s.H_kv, s.D, dtype=torch.bfloat16, device=device))
                      for _ in range(s.layers)]
        order = np.random.default_rng(seed).permutation(num_pages)
        self.free = torch.tensor(order, **i32)
        self.top = torch.tensor([num_pages], **i32)
        self.table = torch.zeros(S, max(held), **i32)
        self.seq_len = torch.zeros(S, **i32)
        self.slots = hpd.ChunkSlots(self.table, self.seq_len, self.free, self.top, max_tokens=room)
        rope = hpd.rope_table(max(self.total) + 64, s.D, device=device)
        self.norm_rope = [hpd.QkNormRope(s.H_q, s.H_kv, s.D, 1 + rand(s.D, std=0.1), 1 + rand(s.D, std=0.1), rope,
                                         sections=s.sections) for _ in range(s.layers)]
        self.attn = [hpd.ChunkAttn(s.H_q, k, v, self.table, max_tokens=room, max_seq_len=max(self.total))
                     for k, v in self.cache]
        # a vision token turns by its row and column, a prompt token by its place
        self.place = torch.zeros(S, max(self.total), 3, **i32)
        for d, ((r, c), n) in enumerate(zip(grids, prompts)):
            y, x = torch.arange(r, **i32), torch.arange(c, **i32)
            self.place[d, : r * c, 1] = y.repeat_interleave(c)
            self.place[d, : r * c, 2] = x.repeat(r)
            self.place[d, r * c: r * c + n] = (max(r, c) + torch.arange(n, **i32))[:, None]
        self.full = torch.tensor(self.vision, **i32)  # vision tokens see all of them
        self.tokens = [rand(n, s.hidden) for n in self.total]
        self.rand = rand

    def step(self, chunk):
        """One step: chunk[d] more tokens of document d through every layer."""
        import torch
        s, done = self.shape, self.seq_len.tolist()
        T = sum(chunk)
        doc = torch.repeat_interleave(torch.arange(len(chunk), device=self.table.device),
                                      torch.tensor(chunk, device=self.table.device))
        x = torch.cat([t[a: a + n] for t, a, n in zip(self.tokens, done, chunk)])
        self.slots(torch.tensor(chunk, dtype=torch.int32, device=self.table.device))
        pos = self.place[doc, self.slots.pos[:T].long()].T.contiguous()
        full = torch.minimum(self.full, self.seq_len)  # (those that have come)
        for i, (k, v) in enumerate(self.cache):
            q = self.norm_rope[i](x @ self.w_in[i], pos, self.slots.slot, k, v)
            out, _ = self.attn[i](q, self.slots.chunk_cu, self.seq_len, full)
            x = x + out.flatten(1) @ self.w_out[i]
        return x

    def prefill(self, per_step):
        """Everything, up to per_step tokens of each document a step, and no more
        than a step has room for; a document's vision tokens, which see one
        another, come in one piece.  Returns the last hidden states of each
        document's tokens."""
        import torch
        got, done = [[] for _ in self.total], [0] * len(self.total)
        while done != self.total:
            chunk, left = [], self.room
            for d, n in enumerate(self.total):
                want = max(min(per_step, n - done[d], left), self.vision[d] - done[d])
                chunk.append(want if want <= left else 0)
                left -= chunk[-1]
            if not any(chunk):
                raise ValueError("a step has no room for a document's vision tokens")
            for rows, part in zip(got, self.step(chunk).split(chunk)):
                rows.append(part)
            done = [a + n for a, n in zip(done, chunk)]
        self.check()
        return [torch.cat(rows) for rows in got]

    def branches(self, per_doc, m, layer=0):
        """One decode step of per_doc branches of each document, m draft tokens
        each, in a layer: returns the BranchAttn call."""
        import torch
        s, dev = self.shape, self.table.device
        S, B = len(self.total), len(self.total) * per_doc
        i32 = dict(dtype=torch.int32, device=dev)
        own = hpd.ChunkSlots(torch.zeros(B, -(-m // PAGE), **i32), torch.zeros(B, **i32), self.free, self.top,
                             max_tokens=B * m)
        own(torch.full((B,), m, **i32))
        prefix = self.seq_len.repeat_interleave(per_doc)
        # (behind the prompt: its last place and one more, the same on every axis)
        last = self.place[torch.arange(S, device=dev), (self.seq_len - 1).long()].amax(-1).repeat_interleave(per_doc * m)
        pos = (last + 1 + own.pos).expand(3, -1).contiguous()
        k, v = self.cache[layer]
        q = self.norm_rope[layer](self.rand(B * m, s.hidden) @ self.w_in[layer], pos, own.slot, k, v)
        cu = torch.zeros(S + 1, **i32)
        cu[1:] = self.seq_len.cumsum(0)
        op = hpd.BranchAttn(hpd.DeviceInputs(
            q=q, prefix_k=None, prefix_v=None, prefix_cu=cu, branch_cu=torch.arange(0, B + 1, per_doc, **i32),
            branch_prefix_len=prefix, k_cache=k, v_cache=v, page_table=own.page_table, branch_len=own.seq_len,
            n_docs=S, B=B, m=m, H_q=s.H_q, H_kv=s.H_kv, D=s.D, num_pages=k.shape[0],
            max_pages=own.page_table.shape[1], prefix_tokens=sum(self.total), max_prefix_len=max(self.total),
            scale=0.0, prefix_page_table=self.table, max_prefix_pages=self.table.shape[1]))
        op()
        if own.errors() or op.errors():
            raise RuntimeError(f"errors on the device: {own.errors():#x} {op.errors():#x}")
        return op

    def check(self):
        err = self.slots.errors()
        for op in self.norm_rope + self.attn:
            err |= op.errors()
        if err:
            raise RuntimeError(f"errors on the device: {err:#x}")


def main():
    import torch
    pages = Pages(Shape(), grids=[(24, 20), (30, 31), (8, 8)], prompts=[40, 17, 200], room=1200)
    hidden = pages.prefill(per_step=256)
    op = pages.branches(per_doc=8, m=4)
    torch.cuda.synchronize()
    print(f"prefilled {sum(pages.total)} tokens of {len(hidden)} documents into "
          f"{pages.cache[0][0].shape[0] - int(pages.top)} pages; one decode step of {op.d.B} branches: "
          f"out {tuple(op.out.shape)}, finite {bool(torch.isfinite(op.out.float()).all())}")


if __name__ == "__main__":
    main()
