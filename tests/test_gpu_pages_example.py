"""The operators on pages together, as examples/serve_pages.py runs them: every turn's attention against a plain one in 64 bits over the
rows that the requests were given, taken to 4 bits by the plain rule; and a turn inside a HIP graph."""
import importlib.util
import math
import os

import pytest
import torch

import pages_util as pu
from paper_2406_05317_amd import binding as lb
from test_gpu_pages import arrays_of, check_attn, make_batch, run_attn

pytestmark = pytest.mark.gpu

PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "serve_pages.py")


def load_example():
    spec = importlib.util.spec_from_file_location("serve_pages", PATH)
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


def test_example_serves_what_it_stored():
    ex = load_example()
    turns = []

    def on_turn(what, r, q, k, v, o):
        """The turn's own rows are in the pages as the rule has them, and the attention is that of the pages."""
        starts, held, tables = r.starts.tolist(), r.held.tolist(), r.tables.cpu()
        R, H = r.pages.c.page_rows, r.pages.c.n_kv_heads
        arrays = arrays_of(r.pages)
        flat = [x.cpu().transpose(0, 1).reshape(H, -1, ex.D) for x in (k, v)]
        for i in range(r.n):
            for x in range(starts[i], starts[i + 1]):
                j = held[i] - (starts[i + 1] - x)
                page = int(tables[i, j // R])
                for y, codes, scales in ((flat[0], *arrays[:2]), (flat[1], *arrays[2:])):
                    want = pu.values(*pu.four_bits(y[:, x]))
                    got = torch.stack([pu.page_values(codes, scales, page, h, j % R) for h in range(H)])
                    assert torch.equal(got, want)
        check_attn(r.pages, q, tables, r.starts.cpu(), r.held.cpu(), o)
        own = [int(p) for h, t in zip(held, tables) for p in t[:-(-h // R)]]
        assert len(own) == len(set(own))
        turns.append(what)

    got = ex.serve(n=5, turns=3, on_turn=on_turn)
    assert turns == ["token"] * 3 + ["message"]
    assert got["held"][0] == 0 and got["held"][1] >= 77 and got["pages_given_back"] > 0


def test_example_tells_and_drops_what_was_refused():
    """Requests whose tables are full are refused turn after turn: counted, not among the tokens served, and zeros in their rows of o."""
    ex = load_example()
    seen = []

    def on_turn(what, r, q, k, v, o):
        at = r.slots.tolist()
        starts, held = r.starts.tolist(), r.held.tolist()
        gone = [i for i in range(r.n) if any(at[x] < 0 for x in range(starts[i], starts[i + 1]))]
        for i in gone:
            assert all(at[x] < 0 for x in range(starts[i], starts[i + 1]))      # as a whole
            held[i] = 0                                                         # a plain request that holds nothing: zeros
        seen.append((what, gone))
        if gone or what == "message":
            check_attn(r.pages, q, r.tables.cpu(), r.starts.cpu(), torch.tensor(held, dtype=torch.int32), o)

    got = ex.serve(n=3, turns=66, rows_each=320, on_turn=on_turn)               # 256 slots of memory and 64 rows behind them
    want = sum(len(gone) for _, gone in seen)
    assert got["refused"] == want > 0 and seen[0][1] == [] and seen[-2][1] != [] and seen[-1][0] == "message"
    assert got["tokens"] == 3 * 66 - sum(len(gone) for what, gone in seen if what == "token")
    assert max(got["held"]) <= 320


def test_turn_in_a_graph():
    """Plan, store and attention of a turn, captured once and replayed with other lengths, rows and queries in the same arrays."""
    pages, q, tables, starts, held = make_batch(7, torch.bfloat16, 2, 4, 128, 16, [(700, 1), (30, 1), (1500, 1), (1, 1)])
    i32 = dict(dtype=torch.int32, device="cuda")
    n, d = 4, 128
    room = torch.full((n, 4), -1, dtype=torch.int32)
    tables = torch.cat((tables, room), 1).cuda()
    free = sorted(set(range(pages.c.n_pages)) - set(tables.flatten().tolist()))
    ring, ends = torch.tensor(free + [-1] * (pages.c.n_pages - len(free)), **i32), torch.tensor([0, len(free)], device="cuda")
    ins = dict(new=torch.ones(n, **i32), held=held.cuda(), q=q.cuda().contiguous(), k=torch.zeros(1, 2, n, d, dtype=q.dtype, device="cuda"),
               v=torch.zeros(1, 2, n, d, dtype=q.dtype, device="cuda"))
    out = dict(held=torch.zeros(n, **i32), ends=torch.zeros_like(ends), starts=torch.zeros(n + 1, **i32), slots=torch.zeros(n, **i32),
               positions=torch.zeros(n, **i32), totals=torch.zeros(4, **i32), o=torch.zeros_like(ins["q"]))
    ws = lb.pages_workspace(pages, n, n, 1, 2000)

    def turn():
        lb.lococo_pages_plan(pages, ins["new"], ins["held"], tables, ring, ends, out["held"], out["ends"], out["starts"], out["slots"],
                             out["positions"], out["totals"])
        lb.lococo_pages_store(pages, ins["k"], ins["v"], out["slots"])
        lb.lococo_pages_attn(pages, ins["q"], out["o"], tables, out["starts"], out["held"], 1, 2000, ws)

    turn()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        turn()
    for step in range(4):
        g = torch.Generator(device="cuda").manual_seed(step)
        for name in ("q", "k", "v"):
            ins[name].copy_(torch.empty(ins[name].shape, device="cuda").normal_(generator=g))
        ins["held"].copy_(torch.tensor([[699, 29, 1499, 0], [300, 29, 1000, 0], [0, 17, 1499, 0], [64, 0, 1, 0]][step]))
        graph.replay()
        torch.cuda.synchronize()
        got = {k: v.clone() for k, v in out.items()}
        turn()
        torch.cuda.synchronize()
        for k in out:                          # (rows that nobody stored, which some of these lengths take in, are NaN)
            torch.testing.assert_close(got[k], out[k], rtol=0, atol=0, equal_nan=True)
        check_attn(pages, ins["q"], tables.cpu(), out["starts"].cpu(), out["held"].cpu(), got["o"])
