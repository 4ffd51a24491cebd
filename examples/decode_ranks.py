"""Decoding with each sequence's cache split over P virtual ranks.

Rank r holds every P-th page of a sequence's keys and values, in 8 bits.  A step rotates the new
token's query and key, writes key and value into the cache of the rank whose turn it is, lets
each rank attend to its own rows, and joins the ranks' partial results: with lse_r the log of a
rank's sum of weights and o_r its output,

    m = max_r lse_r             (an Allreduce, max)
    o = sum_r e^(lse_r - m) o_r / sum_r e^(lse_r - m)     (an Allreduce, sum, of both sums)

which is the attention over all rows.  Run: python -m examples.decode_ranks [ranks] [steps]
"""

from __future__ import annotations

import sys

import torch

from paper_2004_09362_gb300 import gar


class RankedCache:
    """The caches of P ranks for one layer and a batch of sequences of up to `most` tokens."""

    def __init__(self, ranks, batch, q_heads, kv_heads, dim, most, page_size=16, kind=torch.int8):
        self.ranks, self.batch, self.page_size = ranks, batch, page_size
        pages = -(-most // (page_size * ranks))              # of a sequence, at a rank
        shape = (batch * pages, kv_heads, page_size, dim)
        scaled = kind in (torch.int8, torch.float8_e4m3fn)
        self.caches, self.plans = [], []
        for _ in range(ranks):
            k, v = (torch.zeros(shape, dtype=kind, device="cuda") for _ in range(2))
            scales = [torch.zeros(shape[:3], device="cuda") for _ in range(2 if scaled else 0)]
            self.caches.append(gar.KVCache(k, v, *scales))
            self.plans.append(gar.gar_attn_plan_create(q_heads, kv_heads, dim))
        self.page_table = torch.arange(batch * pages, dtype=torch.int32, device="cuda").view(batch, pages)
        self.rope = gar.gar_rope_table(most, gar.gar_rope_frequencies(dim)[0])
        n = batch * q_heads
        self.partial = torch.empty((ranks, batch, q_heads, dim), device="cuda")
        self.lse = torch.empty((ranks, n + -n % 4), device="cuda")      # rows of a multiple of 16 bytes
        self.top = torch.empty_like(self.lse)
        self.sums = torch.empty((ranks, batch, q_heads, dim + 4), device="cuda")
        self.max_plan = gar.gar_plan_create(ranks, self.lse.shape[1], "f32", "max", gar.GAR_STEPS_LO)
        self.sum_plan = gar.gar_plan_create(ranks, self.sums[0].numel(), "f32", "sum", gar.GAR_STEPS_LO)

    def step(self, q, k, v, positions):
        """Attention [batch, q_heads, dim] (float32) of the tokens at `positions` (int64 [batch]), whose keys
        and values become part of the cache."""
        turn = positions // self.page_size                   # the sequence's page, and its rank
        rank, page = turn % self.ranks, turn // self.ranks
        row = positions % self.page_size
        slots = self.page_table.gather(1, page[:, None])[:, 0].long() * self.page_size + row
        q = gar.gar_rope(q, positions, self.rope)
        batch, q_heads = q.shape[:2]
        n = batch * q_heads
        self.lse.fill_(float("-inf"))
        for r, cache in enumerate(self.caches):
            gar.gar_kv_write(cache, k, v, torch.where(rank == r, slots, -1), positions, self.rope)
            # rows of this rank: its whole pages, and what the last one has
            whole = (turn - r + self.ranks - 1) // self.ranks
            rows = whole * self.page_size + torch.where(rank == r, row + 1, 0)
            gar.gar_decode_attention(self.plans[r], q, cache, self.page_table, rows.to(torch.int32), out=self.partial[r],
                                     lse=self.lse[r, :n].view(batch, q_heads))
        self.top.copy_(self.lse)
        gar.gar_allreduce(self.max_plan, self.top, "fused")
        weight = torch.exp(self.lse - self.top)[:, :n].view(self.ranks, batch, q_heads, 1)
        torch.mul(self.partial, weight, out=self.sums[..., :-4])
        self.sums[..., -4:] = weight
        gar.gar_allreduce(self.sum_plan, self.sums.view(self.ranks, -1), "fused")
        return self.sums[0, ..., :-4] / self.sums[0, ..., -1:]      # every rank has it


def main(ranks=6, steps=100, batch=3, q_heads=32, kv_heads=8, dim=128):
    torch.manual_seed(0)
    split = RankedCache(ranks, batch, q_heads, kv_heads, dim, steps)
    whole = RankedCache(1, batch, q_heads, kv_heads, dim, steps)
    worst = 0.0
    for i in range(steps):
        positions = torch.full((batch,), i, dtype=torch.int64, device="cuda")
        q, k, v = (torch.randn(batch, h, dim, device="cuda").bfloat16() for h in (q_heads, kv_heads, kv_heads))
        a, b = split.step(q, k, v, positions), whole.step(q, k, v, positions)
        worst = max(worst, float((a - b).abs().max() / b.abs().max()))
    for cache in split.caches:
        gar.gar_kv_status(cache)
    print(f"{steps} tokens of {batch} sequences over {ranks} ranks: off the undivided cache's by {worst:.1e} at most")
    return worst


if __name__ == "__main__":
    main(*(int(x) for x in sys.argv[1:3]))
