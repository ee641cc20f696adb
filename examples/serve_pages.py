"""Requests of different lengths on one attention layer: compressed prompts, then token by token in 4 bits.

Each request's prompt is scanned by lococo_sequence_forward, which leaves a memory of M slots whatever its length.  The memories go to
pages of 4-bit rows (lococo_pages_plan hands out the pages, lococo_pages_store fills them).  From then on every turn serves all
requests at once: a token each, or a user's next message; one plan, one store and one attention call, no matter how the lengths differ.
A request that ends gives its pages back in the same plan, and a new one takes its place.

    python examples/serve_pages.py [--requests 32] [--turns 64]

Q, K and V are drawn, as a model's projections would give them; nothing is copied to the host between turns.
"""
from __future__ import annotations

import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2406_05317_amd import binding as lb  # noqa: E402

HEADS, KV, D, M, BLOCK, WIDTH = 32, 8, 128, 256, 256, 15
DTYPE = torch.bfloat16


class Requests:
    """The pages of `n` requests and what a turn's plan reads and writes."""

    def __init__(self, n: int, page_rows: int = 64, rows_each: int = 4096):
        per = -(-rows_each // page_rows)
        self.n, self.most = n, per * page_rows
        self.pages = lb.Pages(dtype=DTYPE, n_q_heads=HEADS, n_kv_heads=KV, head_dim=D, page_rows=page_rows, n_pages=n * per)
        self.ring, self.ends = self.pages.fresh_ring()
        i32 = dict(dtype=torch.int32, device="cuda")
        self.tables = torch.full((n, per), -1, **i32)
        self.held, self.starts, self.totals = torch.zeros(n, **i32), torch.zeros(n + 1, **i32), torch.zeros(4, **i32)
        self.next_held, self.next_ends = torch.zeros_like(self.held), torch.zeros_like(self.ends)
        self.sums = torch.zeros(4, dtype=torch.int64, device="cuda")    # over all turns: rows placed, pages taken, given back, refusals
        self.longest = 0                                # what the host knows of the lengths: enough to deal out the work

    def plan(self, new_rows: torch.Tensor, tokens: int, max_new: int):
        """Places new_rows[i] rows (-1: request i ends) of every request; returns the slots and positions of the call's `tokens` rows.  The
        rows of a request that was refused, its table or the pool being full, have no slots (-1)."""
        slots, positions = (torch.empty(tokens, dtype=torch.int32, device="cuda") for _ in range(2))
        lb.lococo_pages_plan(self.pages, new_rows, self.held, self.tables, self.ring, self.ends, self.next_held, self.next_ends, self.starts,
                             slots, positions, self.totals)
        self.held, self.next_held = self.next_held, self.held
        self.ends, self.next_ends = self.next_ends, self.ends
        self.longest = min(self.longest + max_new, self.most)
        self.slots = slots
        self.sums += self.totals                        # (on the device, as everything here)
        return slots, positions

    def attend(self, q, o, max_new: int, workspace):
        """Attention of the planned rows; zeros for those of refused requests, whose attention has no meaning."""
        lb.lococo_pages_attn(self.pages, q, o, self.tables, self.starts, self.held, max_new, self.longest, workspace)
        self.drop(o, self.slots)

    @staticmethod
    def drop(o, slots):
        o.masked_fill_((slots < 0).view(o.shape[0], 1, o.shape[2], 1), 0)

    def workspace(self, tokens: int, max_new: int):
        return lb.pages_workspace(self.pages, self.n, tokens, max_new, self.most)


def compress(prompt_k, prompt_v, q, filters):
    """The memory [1, KV, M, D] that the scan of a prompt leaves, with its number of live slots."""
    cfg = lb.make_config(dtype=DTYPE, batch=1, n_q_heads=HEADS, n_kv_heads=KV, head_dim=D, M=M, conv_width=WIDTH)
    cache, o = lb.Cache(cfg), torch.empty_like(q)
    lb.lococo_sequence_forward(cfg, q, prompt_k, prompt_v, o, filters, None, cache, BLOCK, lb.workspace(cfg, q.shape[2], BLOCK, history=True))
    return cache.k, cache.v, cache.len


def serve(n: int = 32, turns: int = 64, seed: int = 0, on_turn=None, rows_each: int = 4096) -> dict:
    """Runs the requests; on_turn(what, requests, q, k, v, o) is called behind every attention (tests look in there)."""
    g = torch.Generator(device="cuda").manual_seed(seed)

    def rows(heads, b, t, gain):
        return torch.empty((b, heads, t, D), device="cuda").normal_(0.0, gain, generator=g).to(DTYPE)

    filters = torch.empty((M, D, WIDTH), device="cuda").normal_(0.0, (D * WIDTH) ** -0.5, generator=g).to(DTYPE)
    r = Requests(n, rows_each=rows_each)
    # prompts of odd lengths, one after the other; their memories into pages, all in one plan and one store
    memories = [compress(rows(KV, 1, t, D ** -0.5), rows(KV, 1, t, D ** -0.5), rows(HEADS, 1, t, D ** -0.5), filters)
                for t in (100 + (i * 397) % 2500 for i in range(n))]
    live = [m[2] for m in memories]
    new = torch.tensor(live, dtype=torch.int32, device="cuda")
    slots, _ = r.plan(new, sum(live), M)
    lb.lococo_pages_store(r.pages, torch.cat([m[0][:, :, :m[2]] for m in memories], 2), torch.cat([m[1][:, :, :m[2]] for m in memories], 2), slots)

    one = torch.ones(n, dtype=torch.int32, device="cuda")
    ws, o = r.workspace(n, 1), torch.zeros((n, HEADS, 1, D), dtype=DTYPE, device="cuda")
    r.drop(o, slots[:n])                                # (a first call loads torch's kernels)
    prompts = r.sums.clone()
    torch.cuda.synchronize()
    began = time.perf_counter()
    for _ in range(turns):                              # a token each; [n, heads, 1, d] as a decoding batch has them
        q, k, v = rows(HEADS, n, 1, 1.0), rows(KV, n, 1, 1.0), rows(KV, n, 1, 1.0)
        slots, _ = r.plan(one, n, 1)
        lb.lococo_pages_store(r.pages, k, v, slots)
        r.attend(q, o, 1, ws)
        if on_turn:
            on_turn("token", r, q, k, v, o)
    torch.cuda.synchronize()
    seconds = time.perf_counter() - began
    served = int((r.sums - prompts)[0])                 # tokens of requests that were not refused

    # request 0 ends, request 1 gets the user's next message, the others a token
    message = 77
    new = one.clone()
    new[0], new[1] = -1, message
    tokens = message + n - 2
    q, k, v = rows(HEADS, 1, tokens, 1.0), rows(KV, 1, tokens, 1.0), rows(KV, 1, tokens, 1.0)
    slots, _ = r.plan(new, tokens, message)
    lb.lococo_pages_store(r.pages, k, v, slots)
    o = torch.empty_like(q)
    r.attend(q, o, message, r.workspace(tokens, message))
    if on_turn:
        on_turn("message", r, q, k, v, o)
    torch.cuda.synchronize()
    return {"tokens_per_s": served / seconds, "tokens": served, "refused": int(r.sums[3]), "us_per_turn": seconds / turns * 1e6,
            "memory_rows": sum(live), "pages_given_back": int(r.totals[2]), "held": r.held.tolist(),
            "bytes_a_row": 2 * KV * (D // 2 + D // 32), "bytes_a_row_bf16": 2 * KV * D * 2}


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--requests", type=int, default=32)
    ap.add_argument("--turns", type=int, default=64)
    a = ap.parse_args()
    for key, value in serve(a.requests, a.turns).items():
        print(f"{key}: {value}")
