"""Turns with drafted trees on the GPU against plain implementations in 64 bits: positions and masks (equal), attention under masks (the
tolerances of test_gpu_pages.py: the same kernels, other visibility), what is kept and moved (equal), and whole turns."""
import math
import random

import pytest
import torch

import pages_util as pu
import rotate_util as ru
from paper_2406_05317_amd import binding as lb
from test_gpu_pages import arrays_of, make_batch

pytestmark = pytest.mark.gpu
I32 = dict(dtype=torch.int32, device="cuda")


def signed(rows):
    return [[w - (1 << 32) if w >= 1 << 31 else w for w in row] for row in rows]


def words_tensor(rows):
    return torch.tensor(signed(rows), dtype=torch.int32)


def draw_parents(r, w, kind):
    if kind == "chain":
        return list(range(-1, w - 1))
    if kind == "roots":
        return [-1] * w
    if kind == "star":
        return [-1] + [0] * (w - 1)
    return [r.randint(-1, x - 1) if r.random() < 0.8 else x - 1 for x in range(w)]


# ---- positions and masks
@pytest.mark.parametrize("words", [1, 2, 3, 4, 5, 8])
@pytest.mark.parametrize("kind", ["random", "chain", "roots", "star"])
def test_tree(words, kind):
    r = random.Random(words)
    most = 32 * words
    news = [0, 1, most, most - 1, 2, 0, most // 2 + 1, most + 3, 7]     # one request with more rows than a mask names
    pad = 5
    starts = [sum(news[:i]) for i in range(len(news) + 1)]
    held = [w + r.choice([0, 1, 70000]) for w in news]
    parents = [p for w in news for p in draw_parents(r, w, kind)] + [3] * pad
    tokens = len(parents)
    masks, positions = torch.full((tokens, words), 77, **I32), torch.full((tokens,), 77, **I32)
    lb.lococo_pages_tree(torch.tensor(starts, **I32), torch.tensor(held, **I32), torch.tensor(parents, **I32), masks, positions)
    want_m, want_p = ru.tree(starts, held, parents, words, tokens)
    assert positions.tolist() == want_p and masks.tolist() == signed(want_m)
    bases = [r.randint(0, 10 ** 6) for _ in news]
    bases[1] = -5
    lb.lococo_pages_tree(torch.tensor(starts, **I32), torch.tensor(held, **I32), torch.tensor(parents, **I32), masks, positions,
                         torch.tensor(bases, **I32))
    want_m, want_p = ru.tree(starts, held, parents, words, tokens, bases)
    assert positions.tolist() == want_p and masks.tolist() == signed(want_m)


def test_trees_of_numbers_that_make_no_sense():
    """Parents that are no earlier row, rows ahead of the first request, more rows than held, many requests."""
    parents = [9, 0, 1, 5, -7, 2 ** 31 - 1, -2 ** 31, 3, 1, 0, 0]
    starts, held = [2, 6, 6, 10], [4, -3, 1]
    masks, positions = torch.full((11, 1), 77, **I32), torch.full((11,), 77, **I32)
    lb.lococo_pages_tree(torch.tensor(starts, **I32), torch.tensor(held, **I32), torch.tensor(parents, **I32), masks, positions)
    want_m, want_p = ru.tree(starts, held, parents, 1, 11)
    assert positions.tolist() == want_p and masks.tolist() == signed(want_m)
    r = random.Random(3)
    news = [r.choice([0, 1, 5, 30]) for _ in range(4096)]
    starts = [sum(news[:i]) for i in range(4097)]
    parents = [p for w in news for p in draw_parents(r, w, "random")] + [0] * 9000
    held = [w + r.randint(0, 99) for w in news]
    masks, positions = torch.full((len(parents), 1), 77, **I32), torch.full((len(parents),), 77, **I32)
    lb.lococo_pages_tree(torch.tensor(starts, **I32), torch.tensor(held, **I32), torch.tensor(parents, **I32), masks, positions)
    want_m, want_p = ru.tree(starts, held, parents, 1, len(parents))
    assert positions.tolist() == want_p and masks.tolist() == signed(want_m)
    # starts that run backwards or leave the call: no row beside it is touched
    wild = torch.full((64, 1), 77, **I32)
    pos = torch.full((64,), 77, **I32)
    lb.lococo_pages_tree(torch.tensor([5, 2 ** 31 - 1, -4, 40], **I32), torch.tensor([9, 9, 9], **I32), torch.zeros(48, **I32), wild[8:56], pos[8:56])
    assert (wild[:8] == 77).all() and (wild[56:] == 77).all() and (pos[:8] == 77).all() and (pos[56:] == 77).all()


# ---- attention under masks
def run_attn(pages, q, tables, starts, held, masks, o=None, fill=5.0, hint=None):
    """hint: another max_held than the requests' own, which only says how the work is dealt out (tables are made to hold as many)."""
    news = (starts[1:] - starts[:-1]).tolist()
    o = torch.full_like(q, fill, device="cuda") if o is None else o
    if hint:
        wide = torch.full((tables.shape[0], max(tables.shape[1], hint // pages.c.page_rows)), -1, dtype=torch.int32)
        wide[:, :tables.shape[1]] = tables
        ws = lb.pages_workspace(pages, len(held), q.shape[0] * q.shape[2], max(max(news), -(-q.shape[2] // len(held))), hint)
        ws.fill_(255)
        lb.lococo_pages_attn_tree(pages, q.cuda() if not q.is_cuda else q, o, wide.cuda(), starts.cuda(), held.cuda(), words_tensor(masks).cuda(),
                                  max(max(news), -(-q.shape[2] // len(held))), hint, ws)
        return o
    most, tokens = int(held.clamp(min=0).max()), q.shape[0] * q.shape[2]
    promise = max(max(news), -(-tokens // len(held)))
    ws = lb.pages_workspace(pages, len(held), tokens, promise, most)
    if ws is not None:
        ws.fill_(255)                                                  # what a workspace holds before a call may be anything
    lb.lococo_pages_attn_tree(pages, q.cuda() if not q.is_cuda else q, o, tables.cuda(), starts.cuda(), held.cuda(), words_tensor(masks).cuda(),
                              promise, most, ws)
    return o


def check_attn(pages, q, tables, starts, held, masks, got, scale=None):
    b, H, t, d = q.shape
    c = pages.c
    flat = q.cpu().transpose(0, 1).reshape(H, b * t, d)
    o, mass, size = ru.attention(flat, tables, starts.tolist(), held.tolist(), masks, arrays_of(pages), c.page_rows, H // c.n_kv_heads,
                                 scale or 1.0 / math.sqrt(d))
    got = got.cpu().double().transpose(0, 1).reshape(H, b * t, d)
    n = max(1, int(held.max()))
    rel = 4 * (d + 8) * 2.0 ** -23 * size[..., None] + (n + 64) * 2.0 ** -23
    if q.dtype == torch.bfloat16:
        rel = rel + 2.0 ** -8
    first, real = starts.tolist()[0], starts.tolist()[-1]
    o, got, tol = o[:, first:real], got[:, first:real], (rel * mass)[:, first:real] + 1e-30
    assert torch.equal(torch.isnan(o), torch.isnan(got))
    bad = ~((got - o).abs() <= tol) & ~torch.isnan(o)
    assert not bad.any(), (bad.nonzero()[:5].tolist(), ((got - o).abs() / tol)[bad].max().item())


def masks_of(seed, starts, held, words, kind="random"):
    """trees, or (kind "any") masks of any bits, some rows with none"""
    r = random.Random(seed)
    starts, held = starts.tolist(), held.tolist()
    T = starts[-1]
    if kind == "any":
        return [[r.choice([0, 0xffffffff, r.getrandbits(32)]) for _ in range(words)] if r.random() < 0.8 else [0] * words for _ in range(T)]
    parents = [p for a, b in zip(starts, starts[1:]) for p in draw_parents(r, b - a, kind)]
    return ru.tree(starts, held, parents, words, T)[0]


SHAPES = [  # kv, group, d, R
    (2, 1, 128, 64), (1, 4, 128, 16), (2, 3, 64, 32), (1, 8, 64, 128), (1, 16, 128, 64), (2, 2, 96, 16), (1, 5, 256, 64), (1, 1, 32, 1024)]
LENGTHS = [
    [(1, 1)], [(16, 16), (17, 3), (300, 2), (64, 64), (65, 33)], [(5, 5), (3, 3), (40, 0), (100, 1), (0, 0), (129, 40)],
    [(0, 3), (2, 5), (200, 70)],                                       # nothing held, fewer rows than queries
    [(700, 130), (131, 130), (150, 90)]]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("kv,group,d,R", SHAPES)
@pytest.mark.parametrize("lens", range(len(LENGTHS)))
@pytest.mark.parametrize("kind", ["random", "any"])
def test_attention(dtype, kv, group, d, R, lens, kind):
    print(dtype, kv, group, d, R, LENGTHS[lens], kind, flush=True)
    batch = make_batch(lens, dtype, kv, group, d, R, LENGTHS[lens])
    words = max(1, -(-max(w for _, w in LENGTHS[lens]) // 32))
    masks = masks_of(lens, batch[3], batch[4], words, kind)
    check_attn(*batch, masks, run_attn(*batch, masks))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("kv,group,d,R,lens", [
    (2, 4, 128, 64, [(5000, 5), (9, 9), (1023, 3)]), (1, 1, 128, 16, [(9001, 12)]), (1, 2, 64, 32, [(4097, 7), (2500, 60)]),
    (1, 4, 128, 64, [(3000, 40), (10, 3)]), (2, 1, 64, 128, [(2100, 90)])])
@pytest.mark.parametrize("kind", ["random", "any"])
def test_attention_over_long_contexts(dtype, kv, group, d, R, lens, kind):
    """Lengths where the rows of one request are shared out between workgroups and their results joined."""
    batch = make_batch(11, dtype, kv, group, d, R, lens)
    masks = masks_of(12, batch[3], batch[4], -(-max(w for _, w in lens) // 32), kind)
    check_attn(*batch, masks, run_attn(*batch, masks))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("kv,group,d", [(2, 4, 128), (1, 2, 64), (2, 2, 96)])
@pytest.mark.parametrize("lens", [[(60, 1), (300, 20)], [(2500, 40), (70, 70)], [(900, 130), (64, 64), (33, 1)]])
def test_a_chain_is_causal_attention(dtype, kv, group, d, lens):
    """Every row the child of the one ahead: the visibility of lococo_pages_attn, whose results (sums in another order) both are held to."""
    pages, q, tables, starts, held = make_batch(41, dtype, kv, group, d, 16, lens)
    masks = masks_of(0, starts, held, -(-max(w for _, w in lens) // 32), "chain")
    check_attn(pages, q, tables, starts, held, masks, run_attn(pages, q, tables, starts, held, masks))
    o = torch.full_like(q, 5.0, device="cuda")
    ws = lb.pages_workspace(pages, len(lens), q.shape[2], max(w for _, w in lens), int(held.max()))
    lb.lococo_pages_attn(pages, q.cuda(), o, tables.cuda(), starts.cuda(), held.cuda(), max(w for _, w in lens), int(held.max()), ws)
    check_attn(pages, q, tables, starts, held, masks, o)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("d", [64, 128, 96])
@pytest.mark.parametrize("held,new", [(200, 50), (2000, 40), (50, 50), (1100, 5)])
def test_attention_keeps_nan_where_it_is_seen(dtype, d, held, new):
    """A marked block of K reaches every query whose mask sees its row, one of V those queries' 32 columns, and no query beside them."""
    R = 16
    pages, q, tables, starts, hl = make_batch(31, dtype, 2, 2, d, R, [(held, new), (90, new), (held - 3, new)])
    mark = lambda s, i, r, h, c: s.__setitem__((int(tables[i, r // R]), h, c, r % R), 255)
    mark(pages.v_scales, 0, held - new + 2, 1, 1)                       # a new row of request 0
    mark(pages.v_scales, 0, held - 1, 0, 0)
    if new < 90:
        mark(pages.v_scales, 1, 90 - new - 1, 0, 0)                     # the last row ahead of request 1's new ones: all see it
    mark(pages.k_scales, 2, held - 3 - new + 3, 0, 1)                   # a new row of request 2
    words = -(-new // 32)
    for kind in ("random", "any"):
        masks = masks_of(5, starts, hl, words, kind)
        got = run_attn(pages, q, tables, starts, hl, masks)
        assert torch.isnan(got).any() and not torch.isnan(got).all()
        check_attn(pages, q, tables, starts, hl, masks, got)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("d", [64, 128, 96])
def test_rows_that_see_nothing(dtype, d):
    """No rows ahead and empty masks: zeros; masks that name rows behind the request's last: none of them."""
    batch = make_batch(51, dtype, 1, 2, d, 16, [(40, 40), (7, 7), (100, 3)])
    masks = [[0, 0] for _ in range(50)]
    got = run_attn(*batch, masks)
    assert not got[:, :, :47].any() and got[:, :, 47:].any()
    check_attn(*batch, masks, got)
    masks = [[0xffffffff, 0xffffffff] for _ in range(50)]
    check_attn(*batch, masks, run_attn(*batch, masks))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("d", [64, 128, 96])
def test_masks_shorter_than_the_requests(dtype, d):
    """New rows that a mask has no bits for are seen by nobody."""
    batch = make_batch(52, dtype, 1, 2, d, 16, [(90, 70), (40, 33), (1000, 40)])
    masks = masks_of(1, batch[3], batch[4], 1, "any")
    check_attn(*batch, masks, run_attn(*batch, masks))
    pages, q, tables, starts, held = make_batch(53, dtype, 1, 1, d, 16, [(400, 300)])          # more than any mask names
    masks = masks_of(2, starts, held, 8, "any")
    check_attn(pages, q, tables, starts, held, masks, run_attn(pages, q, tables, starts, held, masks))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("d", [64, 128, 96])
@pytest.mark.parametrize("held", [300, 2500])
def test_attention_leaves_out_what_is_no_page(dtype, d, held):
    batch = make_batch(61, dtype, 1, 2, d, 16, [(held, 20), (100, 40)])
    tables = batch[2]
    tables[0, 3], tables[0, (held - 5) // 16], tables[1, 4] = -1, 10 ** 9, -1
    masks = masks_of(6, batch[3], batch[4], 2)
    check_attn(*batch, masks, run_attn(*batch, masks))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("d", [64, 128, 96])
def test_views_scale_and_rows_of_nobody(dtype, d):
    """Token-major q and o with gaps, rows of nobody ahead and behind, another scale; nothing beside the rows is written."""
    lens = [(150, 21), (60, 9)]
    pages, _, tables, starts, held = make_batch(62, dtype, 2, 2, d, 32, lens)
    pages.c.attn_scale = 0.3
    starts = starts + 3
    g = torch.Generator().manual_seed(9)
    wide = torch.randn(1, 40, 4, d + 8, generator=g).to(dtype).cuda()
    out = torch.full((1, 40, 4, d + 8), 5.0, dtype=dtype, device="cuda")
    q, o = wide[..., :d].transpose(1, 2), out[..., :d].transpose(1, 2)
    masks = [[0]] * 3 + masks_of(7, starts - 3, held, 1) + [[0xffffffff]] * 7
    run_attn(pages, q, tables, starts, held, masks, o=o)
    check_attn(pages, q, tables, starts, held, masks, o, scale=0.3)
    assert (out[..., d:] == 5.0).all() and (out[:, :3] == 5.0).all() and (out[:, 33:] == 5.0).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("n,group", [(40, 4), (130, 1), (700, 4)])
def test_many_requests_most_of_them_idle(dtype, n, group):
    r = random.Random(n)
    lens = [(r.randint(20, 90), r.randint(1, 20)) if r.random() < 0.1 else (r.randint(0, 50), 0) for _ in range(n)]
    lens[3] = (80, 17)
    batch = make_batch(63, dtype, 1, group, 64, 16, lens)
    masks = masks_of(8, batch[3], batch[4], 1)
    check_attn(*batch, masks, run_attn(*batch, masks))


def test_attention_repeats_bit_for_bit():
    batch = make_batch(64, torch.bfloat16, 4, 4, 128, 64, [(6000, 30), (900, 61), (64, 64)])
    masks = masks_of(9, batch[3], batch[4], 2)
    first = run_attn(*batch, masks)
    for _ in range(3):
        assert torch.equal(first, run_attn(*batch, masks))


# ---- what is kept
def draw_keep(seed, n, R, share, refused=0.1, pad=3):
    r = random.Random(seed)
    news = [r.choice([0, 1, 2, 7, 40, 64, 65, 130]) for _ in range(n)]
    held = [w + r.choice([0, 1, R - 1, R, 3 * R + 2]) for w in news]
    counts = [-(-h // R) for h in held]
    P, width = sum(counts) + 5, max(counts) + 2
    ids = list(range(P))
    r.shuffle(ids)
    tables, slots = [[-1] * width for _ in range(n)], []
    for i, c in enumerate(counts):
        tables[i][:c], ids = ids[:c], ids[c:]
        out = r.random() < refused
        slots += [-1 if out else tables[i][x // R] * R + x % R for x in range(held[i] - news[i], held[i])]
    kept = [r.choice([1, -1, 7]) if r.random() < share else 0 for _ in slots]
    head = r.randrange(50 * P)
    ring = [-1] * P
    for j, p in enumerate(ids):
        ring[(head + j) % P] = p
    starts = [sum(news[:i]) for i in range(n + 1)]
    return dict(P=P, R=R, tables=tables, starts=starts, held=held, slots=slots + [-1] * pad, kept=kept + [1] * pad, ring=ring, ends=[head, head + len(ids)])


def run_keep(c):
    pages = lb.Pages(dtype=torch.bfloat16, n_q_heads=1, n_kv_heads=1, head_dim=32, page_rows=c["R"], n_pages=c["P"])
    t = {k: torch.tensor(c[k], **I32) for k in ("tables", "starts", "held", "slots", "kept", "ring")}
    ends, n, T = torch.tensor(c["ends"], dtype=torch.int64, device="cuda"), len(c["held"]), len(c["slots"])
    ends_after = torch.zeros(2, dtype=torch.int64, device="cuda")
    out = {k: torch.full((m,), -77, **I32) for k, m in dict(held=n, sources=T, targets=T, totals=2).items()}
    lb.lococo_pages_keep(pages, t["tables"], t["starts"], t["held"], t["slots"], t["kept"], t["ring"], ends, out["held"], ends_after, out["sources"],
                         out["targets"], out["totals"])
    return dict({k: v.tolist() for k, v in out.items()}, ends=ends_after.tolist(), ring=t["ring"].tolist())


def want_keep(c):
    return ru.keep(c["P"], c["R"], c["tables"], c["starts"], c["held"], c["slots"], c["kept"], c["ring"], c["ends"])


@pytest.mark.parametrize("n", [1, 2, 5, 64, 257, 1025, 4096])
@pytest.mark.parametrize("share", [0.0, 0.2, 0.9, 1.0])
@pytest.mark.parametrize("R", [16, 64])
def test_keep(n, share, R):
    c = draw_keep(n + int(10 * share), n, R, share)
    assert run_keep(c) == want_keep(c)


def test_keep_of_nothing_and_of_what_makes_no_sense():
    c = draw_keep(5, 3, 16, 0.5)
    c.update(starts=[0, 0, 0, 0], slots=[], kept=[])
    assert run_keep(c) == want_keep(c)
    c = draw_keep(6, 8, 16, 0.5, refused=0.0)
    c["held"] = [-5, 10 ** 9, 3, 0, 2 ** 31 - 1, c["held"][5], 1, 17]
    assert run_keep(c) == want_keep(c)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("d", [32, 64, 96, 128, 160, 256])
@pytest.mark.parametrize("heads,R,share", [(1, 16, 0.3), (5, 64, 0.9), (8, 16, 1.0), (2, 1024, 0.05)])
def test_move(dtype, d, heads, R, share):
    """Kept rows lie behind each other afterwards, bit for bit; all other rows are as they were."""
    c = draw_keep(d + heads, 9, R, share, refused=0.1)
    if c["P"] * R * heads * d > 1 << 24:
        c = draw_keep(d + heads, 3, R, share)
    pages = lb.Pages(dtype=dtype, n_q_heads=heads, n_kv_heads=heads, head_dim=d, page_rows=R, n_pages=c["P"])
    arrays = (pages.k_codes, pages.k_scales, pages.v_codes, pages.v_scales)
    for x in arrays:
        x.copy_(torch.randint(0, 256, x.shape, dtype=torch.uint8, device="cuda"))
    want = [x.cpu() for x in arrays]
    k = want_keep(c)
    before = [x.clone() for x in want]
    for a, b in zip(k["sources"], k["targets"]):
        if a >= 0:
            for i in (0, 2):
                want[i][b // R, :, b % R] = before[i][a // R, :, a % R]
                want[i + 1][b // R, :, :, b % R] = before[i + 1][a // R, :, :, a % R]
    sources, targets = torch.tensor(k["sources"], **I32), torch.tensor(k["targets"], **I32)
    lb.lococo_pages_move(pages, torch.tensor(c["starts"], **I32), sources, targets)
    for x, y in zip(arrays, want):
        assert torch.equal(x.cpu(), y)
    # slots outside the pages, and rows onto themselves: nothing
    n = c["P"] * R
    bad = torch.tensor([-1, n, 0, 2 ** 31 - 1, 5, 3, -2 ** 31], **I32)
    lb.lococo_pages_move(pages, torch.tensor([0, 7], **I32), bad, torch.tensor([0, 1, -1, 2, 5, n, 4], **I32))
    for x, y in zip(arrays, want):
        assert torch.equal(x.cpu(), y)


# ---- whole turns
class Server:
    """Requests in pages, turn by turn: plan, append, and for trees what is kept."""

    def __init__(self, dtype, n, Hq, Hkv, d, R, n_pages, width, g):
        self.pages = lb.Pages(dtype=dtype, n_q_heads=Hq, n_kv_heads=Hkv, head_dim=d, page_rows=R, n_pages=n_pages)
        self.ring, self.ends = self.pages.fresh_ring()
        self.tables = torch.full((n, width), -1, **I32)
        self.held = torch.zeros(n, **I32)
        freqs = (10000.0 ** (-torch.arange(0, d, 2, dtype=torch.float64) / d)).float().cuda()
        w = [(1 + 0.2 * torch.randn(d, generator=g)).to(dtype).cuda() for _ in range(2)]
        self.rot = lb.Rotation(dtype=dtype, n_q_heads=Hq, n_kv_heads=Hkv, head_dim=d, freqs=freqs, norm=True, q_weight=w[0], k_weight=w[1])
        self.n, self.dtype, self.shape = n, dtype, (Hq, Hkv, d)

    def plan(self, news):
        n, T = self.n, sum(news)
        o = dict(held=torch.empty(n, **I32), ends=torch.empty(2, dtype=torch.int64, device="cuda"), starts=torch.empty(n + 1, **I32),
                 slots=torch.empty(T, **I32), positions=torch.empty(T, **I32), totals=torch.empty(4, **I32))
        lb.lococo_pages_plan(self.pages, torch.tensor(news, **I32), self.held, self.tables, self.ring, self.ends, o["held"], o["ends"], o["starts"],
                             o["slots"], o["positions"], o["totals"])
        assert o["totals"][3] == 0
        self.held, self.ends = o["held"], o["ends"]
        return o

    def attend(self, qkv, o, positions, news, masks=None):
        Hq, Hkv, d = self.shape
        q, k, v = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:]
        qo, out = torch.empty(1, Hq, q.shape[2], d, dtype=self.dtype, device="cuda"), torch.empty(1, Hq, q.shape[2], d, dtype=self.dtype, device="cuda")
        lb.lococo_pages_append(self.pages, self.rot, q, k, v, qo, o["slots"], positions)
        most = int(self.held.max())
        ws = lb.pages_workspace(self.pages, self.n, q.shape[2], max(news), most)
        if masks is None:
            lb.lococo_pages_attn(self.pages, qo, out, self.tables, o["starts"], self.held, max(news), most, ws)
        else:
            lb.lococo_pages_attn_tree(self.pages, qo, out, self.tables, o["starts"], self.held, masks, max(news), most, ws)
        return out

    def rows(self, i):
        """all rows of a request, as they lie"""
        h, R = int(self.held[i]), self.pages.c.page_rows
        page, row = self.tables[i].long()[torch.arange(h, device="cuda") // R], torch.arange(h, device="cuda") % R
        return [x for codes, scales in ((self.pages.k_codes, self.pages.k_scales), (self.pages.v_codes, self.pages.v_scales))
                for x in (codes[page, :, row], scales[page, :, :, row])]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("Hq,Hkv,d,R", [(4, 2, 128, 16), (6, 3, 64, 32), (2, 1, 96, 16)])
def test_drafted_turns_leave_what_one_token_at_a_time_leaves(dtype, Hq, Hkv, d, R):
    """Trees are appended, attended to and thinned out to a path, turn after turn; the same tokens one by one leave the same rows bit for bit
    and the same attention (fp32 sums in another order: the tolerance of a result against itself in 64 bits, twice)."""
    n, g, r = 3, torch.Generator().manual_seed(1), random.Random(2)
    tree, line = (Server(dtype, n, Hq, Hkv, d, R, 60, 14, torch.Generator().manual_seed(7)) for _ in range(2))
    first = [20, 1, 33]
    x = torch.randn(1, Hq + 2 * Hkv, sum(first), d, generator=g).to(dtype).cuda()
    for s in (tree, line):
        p = s.plan(first)
        s.attend(x, p, p["positions"], first)
    free = None
    for turn in range(4):
        news = [r.choice([1, 2, 9, 17, 33]) for _ in range(n)]
        T, words = sum(news), 2
        p = tree.plan(news)
        parents = [q for w in news for q in draw_parents(r, w, "random")]
        masks, positions = torch.empty(T, words, **I32), torch.empty(T, **I32)
        lb.lococo_pages_tree(p["starts"], tree.held, torch.tensor(parents, **I32), masks, positions)
        x = torch.randn(1, Hq + 2 * Hkv, T, d, generator=g).to(dtype).transpose(1, 2).contiguous().transpose(1, 2).cuda()
        got = tree.attend(x, p, positions, news, masks)
        # a path: some row and all it continues
        kept, paths, at = [0] * T, [], 0
        for w in news:
            up, path = r.randrange(w), []
            while up >= 0:
                path.append(up)
                up = parents[at + up]
            path.reverse()
            paths.append([at + j for j in path])
            for j in path:
                kept[at + j] = 1
            at += w
        after, ends = torch.empty(n, **I32), torch.empty(2, dtype=torch.int64, device="cuda")
        sources, targets, totals = torch.empty(T, **I32), torch.empty(T, **I32), torch.empty(2, **I32)
        lb.lococo_pages_keep(tree.pages, tree.tables, p["starts"], tree.held, p["slots"], torch.tensor(kept, **I32), tree.ring, tree.ends, after, ends,
                             sources, targets, totals)
        lb.lococo_pages_move(tree.pages, p["starts"], sources, targets)
        tree.held, tree.ends = after, ends
        assert totals[0] == sum(kept)
        # the same tokens one by one
        for step in range(max(map(len, paths))):
            ones = [int(step < len(q)) for q in paths]
            rows = [q[step] for q in paths if step < len(q)]
            p1 = line.plan(ones)
            want = line.attend(x[:, :, rows], p1, p1["positions"], ones)
            a, b = got[:, :, rows].float(), want.float()
            err = 2 * (2.0 ** -8 if dtype == torch.bfloat16 else 0.0) + 2 * (4 * (d + 8) * 40 + 400) * 2.0 ** -23
            assert ((a - b).abs() <= err * (b.abs() + 4.0)).all(), (turn, step)          # sums of p |v| are below 4: values are normal
        assert tree.held.tolist() == line.held.tolist()
        for i in range(n):
            for a, b in zip(tree.rows(i), line.rows(i)):
                assert torch.equal(a, b), (turn, i)
        # no page is lost or held twice
        head, tail = tree.ends.tolist()
        free = [int(tree.ring[j % 60]) for j in range(head, tail)]
        mine = [int(x) for i in range(n) for x in tree.tables[i, :-(-int(tree.held[i]) // R)]]
        assert sorted(free + mine) == list(range(60))


LONG = 1 << 21                                                         # what a caller may say of requests of any length


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("kv,group,d,R", [(2, 1, 128, 64), (1, 4, 128, 16), (2, 3, 64, 32), (1, 16, 128, 64), (1, 8, 64, 128)])
@pytest.mark.parametrize("lens", [[(16, 16), (17, 3), (300, 2), (64, 64), (65, 33)], [(5, 5), (3, 3), (40, 0), (100, 1), (0, 0), (129, 40)],
                                  [(0, 3), (2, 5), (200, 70)], [(700, 130), (131, 130), (550, 90)], [(3000, 9), (513, 40), (512, 40), (511, 40)],
                                  [(4097, 33)]])
@pytest.mark.parametrize("kind", ["random", "any"])
def test_attention_dealt_out_by_lengths(dtype, kv, group, d, R, lens, kind):
    """Said to be long: work is dealt out by a launch ahead, tiles to a wave alone and to four, in one part and in several."""
    print(dtype, kv, group, d, R, lens, kind, flush=True)
    batch = make_batch(101, dtype, kv, group, d, R, lens)
    masks = masks_of(102, batch[3], batch[4], -(-max(w for _, w in lens) // 32), kind)
    got = run_attn(*batch, masks, hint=LONG)
    check_attn(*batch, masks, got)
    assert torch.equal(got, run_attn(*batch, masks, hint=LONG))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("d", [64, 128])
def test_marks_and_missing_pages_where_work_is_dealt_out(dtype, d):
    lens = [(2000, 40), (90, 40), (300, 33), (600, 7)]
    pages, q, tables, starts, held = make_batch(103, dtype, 2, 2, d, 16, lens)
    mark = lambda s, i, r, h, c: s.__setitem__((int(tables[i, r // 16]), h, c, r % 16), 255)
    mark(pages.v_scales, 0, 1962, 1, 1)
    mark(pages.v_scales, 0, 100, 0, 0)
    mark(pages.v_scales, 1, 60, 0, 1)
    mark(pages.k_scales, 2, 270, 1, 0)
    tables[3, 5], tables[0, 50], tables[2, 18] = -1, 10 ** 9, -1
    for kind in ("random", "any"):
        masks = masks_of(7, starts, held, 2, kind)
        got = run_attn(pages, q, tables, starts, held, masks, hint=LONG)
        assert torch.isnan(got).any() and not torch.isnan(got).all()
        check_attn(pages, q, tables, starts, held, masks, got)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("n", [64, 65, 130, 1100])
def test_many_requests_dealt_out(dtype, n):
    """More requests than a workgroup has threads; most of them idle, one long."""
    r = random.Random(n)
    lens = [(r.randint(20, 90), r.randint(1, 20)) if r.random() < 60 / n else (r.randint(0, 50), 0) for _ in range(n)]
    lens[7] = (1500, 30)
    batch = make_batch(104, dtype, 1, 4, 64, 16, lens)
    masks = masks_of(8, batch[3], batch[4], 1)
    check_attn(*batch, masks, run_attn(*batch, masks, hint=LONG))


def test_starts_that_do_not_ascend_touch_nothing_else():
    """Requests that claim each other's rows: whatever is computed, nothing beside the call's rows of o is written."""
    pages, q, tables, starts, held = make_batch(105, torch.bfloat16, 1, 2, 64, 16, [(100, 20), (90, 20), (80, 20)])
    out = torch.full((1, 2, 80, 64), 5.0, dtype=torch.bfloat16, device="cuda")
    bad = torch.tensor([40, 60, 0, 60], dtype=torch.int32)
    for hint in (None, LONG):
        run_attn(pages, q, tables, bad, held, [[0xffffffff]] * 60, o=out[:, :, 10:70], hint=hint)
        assert (out[:, :, :10] == 5.0).all() and (out[:, :, 70:] == 5.0).all()


def test_a_turn_captured():
    """Plan, trees, append, attention, keeping and moving in one graph, replayed with other drafts; an eager run beside it."""
    dtype, n, news, T, words = torch.bfloat16, 4, [7, 1, 12, 5], 25, 1
    runs = [Server(dtype, n, 8, 2, 128, 16, 80, 16, torch.Generator().manual_seed(4)) for _ in range(2)]
    g, r = torch.Generator().manual_seed(5), random.Random(6)
    data = dict(x=torch.randn(1, 12, T, 128, generator=g).to(dtype).cuda(), parents=torch.zeros(T, **I32), kept=torch.zeros(T, **I32),
                new=torch.tensor(news, **I32))

    def buffers(s):
        s.o = dict(held=torch.empty(n, **I32), ends=torch.empty(2, dtype=torch.int64, device="cuda"), starts=torch.empty(n + 1, **I32),
                   slots=torch.empty(T, **I32), positions=torch.empty(T, **I32), totals=torch.empty(4, **I32))
        s.t = dict(masks=torch.empty(T, words, **I32), positions=torch.empty(T, **I32), qo=torch.empty(1, 8, T, 128, dtype=dtype, device="cuda"),
                   out=torch.empty(1, 8, T, 128, dtype=dtype, device="cuda"), sources=torch.empty(T, **I32), targets=torch.empty(T, **I32),
                   totals=torch.empty(2, **I32), held=torch.empty(n, **I32), ends=torch.empty(2, dtype=torch.int64, device="cuda"))
        s.ws = lb.pages_workspace(s.pages, n, T, 12, 256)

    def turn(s):
        o, t = s.o, s.t
        lb.lococo_pages_plan(s.pages, data["new"], s.held, s.tables, s.ring, s.ends, o["held"], o["ends"], o["starts"], o["slots"], o["positions"], o["totals"])
        lb.lococo_pages_tree(o["starts"], o["held"], data["parents"], t["masks"], t["positions"])
        lb.lococo_pages_append(s.pages, s.rot, data["x"][:, :8], data["x"][:, 8:10], data["x"][:, 10:], t["qo"], o["slots"], t["positions"])
        lb.lococo_pages_attn_tree(s.pages, t["qo"], t["out"], s.tables, o["starts"], o["held"], t["masks"], 12, 256, s.ws)
        lb.lococo_pages_keep(s.pages, s.tables, o["starts"], o["held"], o["slots"], data["kept"], s.ring, o["ends"], t["held"], t["ends"], t["sources"],
                             t["targets"], t["totals"])
        lb.lococo_pages_move(s.pages, o["starts"], t["sources"], t["targets"])
        s.held.copy_(t["held"])
        s.ends.copy_(t["ends"])

    for s in runs:
        buffers(s)
    graphed, eager = runs
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        turn(graphed)
    for k in range(6):
        data["x"].copy_(torch.randn(data["x"].shape, generator=g).to(dtype))
        data["parents"].copy_(torch.tensor([q for w in news for q in draw_parents(r, w, "random")], dtype=torch.int32))
        data["kept"].copy_(torch.tensor([int(r.random() < 0.4) for _ in range(T)], dtype=torch.int32))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            turn(eager)
        torch.cuda.synchronize()
        assert torch.equal(graphed.t["out"], eager.t["out"]) and torch.isfinite(eager.t["out"].float()).all()
        assert graphed.held.tolist() == eager.held.tolist() and graphed.ends.tolist() == eager.ends.tolist()
        assert torch.equal(graphed.tables, eager.tables) and torch.equal(graphed.ring, eager.ring)
        for i in range(n):
            for a, b in zip(graphed.rows(i), eager.rows(i)):
                assert torch.equal(a, b), (k, i)


def test_refusals_of_the_binding():
    batch = make_batch(70, torch.bfloat16, 1, 2, 64, 16, [(30, 4), (20, 3)])
    pages, q, tables, starts, held = batch
    args = [tables.cuda(), starts.cuda(), held.cuda()]
    q, o, masks = q.cuda(), torch.empty_like(q, device="cuda"), torch.zeros(7, 1, **I32)
    good = lambda **k: lb.lococo_pages_attn_tree(pages, q, o, *args, k.get("masks", masks), k.get("new", 4), 30, k.get("ws"))
    good()
    for bad in (masks[:6], masks[:, 0], torch.zeros(7, 2, **I32)[:, :1].transpose(0, 1)):
        with pytest.raises((ValueError, TypeError)):
            good(masks=bad)
    with pytest.raises(TypeError):
        good(masks=masks.long())
    with pytest.raises(TypeError):
        good(masks=masks.cpu())
    with pytest.raises(TypeError):
        good(ws=torch.empty(64, dtype=torch.uint8))
    with pytest.raises(lb.LococoError) as e:
        good(masks=torch.zeros(7, 9, **I32))
    assert e.value.status == lb.LOCOCO_EUNSUPPORTED
    with pytest.raises(lb.LococoError) as e:
        good(new=3)
    assert e.value.status == lb.LOCOCO_EINVAL
    with pytest.raises(ValueError):
        lb.lococo_pages_tree(args[1], args[2], torch.zeros(7, **I32), masks, torch.zeros(6, **I32))
    with pytest.raises(ValueError):
        lb.lococo_pages_move(pages, args[1], torch.zeros(7, **I32), torch.zeros(6, **I32))
