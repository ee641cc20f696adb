"""Norm and rotation of rows on the GPU, forward and backward, and rows appended to pages, against plain implementations in 64 bits.

Tolerances, u = 2^-24, per element, from the arithmetic the header promises (fp32, one rounding at the end):
  one over the root: a sum of d squares, (d + 1) u of it, half of that through the root, the root, the division and the mean's: (d / 2 + 4) u
  a normed value: two more products.  Cosines and sines: the angle in half turns is rounded to fp32, pi 2^-25 < 1.6 u, the function's own
  error is some units: 8 u together.  A turned value: two products and a sum, so (d / 2 + 16) u (|n_a| + |n_b|)
  the way back: a turned gradient G with 10 u (|g_a| + |g_b|), times w and one; the row's mean of w G xhat: (d + d / 2 + 24) u of its magnitudes;
  their difference and the factors: (2 d + 48) u of (|w| |G| + |xhat| mean(|w| |G| |xhat|)) one
  a weight's gradient over N rows: (N + d + 32) u sum |G| |xhat|, N in the worst order of adding
  bf16 results: half a step, 2^-8 of the value, beside it."""
import math

import pytest
import torch

import pages_util as pu
import rotate_util as ru
from paper_2406_05317_amd import binding as lb
from test_gpu_pages import arrays_of

pytestmark = pytest.mark.gpu
I32 = dict(dtype=torch.int32, device="cuda")
U = 2.0 ** -24


def make(seed, dtype, b, t, Hq, Hkv, d, r, adjacent, norm, weights, layout="heads", far=5000, nobody=0.0, extra=0):
    """A rotation and raw rows (device) with their positions; extra: further heads in the same projection."""
    g = torch.Generator().manual_seed(seed)
    rows = torch.randn(b, Hq + Hkv + extra, t, d, generator=g) * torch.empty(Hq + Hkv + extra, 1, d).log_normal_(0.0, 0.5, generator=g)
    rows = rows.to(dtype).cuda()
    if layout == "tokens":                                             # as one projection writes them
        rows = rows.transpose(1, 2).contiguous().transpose(1, 2)
    elif layout == "gaps":
        wide = torch.full((b, Hq + Hkv + extra, t + 3, d + 16), 7.0, dtype=dtype, device="cuda")
        wide[:, :, :t, 8:d + 8] = rows
        rows = wide[:, :, :t, 8:d + 8]
    freqs = (10000.0 ** (-torch.arange(0, r, 2, dtype=torch.float64) / max(r, 1))).float().cuda() if r else None
    ws = [None, None]
    if weights != "none":
        ws = [(1 + 0.3 * torch.randn((h, d) if weights == "heads" else (d,), generator=g)).to(dtype).cuda() for h in (Hq, Hkv)]
    rot = lb.Rotation(dtype=dtype, n_q_heads=Hq, n_kv_heads=Hkv, head_dim=d, freqs=freqs, adjacent=adjacent, norm=norm, norm_eps=1e-5,
                      q_weight=ws[0], k_weight=ws[1])
    pos = None
    if far:
        pos = torch.randint(0, far, (b, 1), generator=g) + torch.arange(t)
        pos[torch.rand(b, t, generator=g) < nobody] = -1
        pos = pos.flatten().int().cuda()
    return rot, rows, pos, ws, g


def angle_of(rot, pos, b, t):
    pos = torch.arange(t).repeat(b) if pos is None else pos.cpu()
    if rot.freqs is None:
        return torch.zeros(b, t, 0, dtype=torch.float64)
    return ru.angles(pos.clamp(min=0), rot.freqs.cpu()).reshape(b, t, -1)


EPS = float(torch.tensor(1e-5, dtype=torch.float32))


def check_forward(rot, x, w, pos, got, adjacent, norm, untouched):
    b, H, t, d = x.shape
    x, w, got = x.cpu(), None if w is None else w.cpu(), got.cpu()
    r, ang = rot.c.rotary_dim, angle_of(rot, pos, b, t)
    want = ru.forward(x, w, ang, r, adjacent, norm, EPS)
    n = ru.normed(x, w, norm, EPS)[0]
    tol = (d / 2 + 16) * U * ru.reach(n, r, adjacent)
    if got.dtype == torch.bfloat16:
        tol = tol + 2.0 ** -8 * want.abs()
    real = torch.ones(b, t, dtype=torch.bool) if pos is None else (pos.cpu() >= 0).reshape(b, t)
    real = real[:, None, :, None].expand_as(want)
    assert torch.equal(got[~real], torch.full_like(got[~real], untouched))
    bad = real & ~((got.double() - want).abs() <= tol + 1e-36)
    assert not bad.any(), (bad.nonzero()[:4].tolist(), ((got.double() - want).abs() / tol)[bad].max().item())


KINDS = [  # b, t, Hq, Hkv, d, r, adjacent, norm, weights
    (1, 1, 1, 1, 128, 128, False, True, "shared"), (2, 37, 4, 2, 128, 128, False, True, "heads"), (1, 33, 3, 1, 64, 32, True, True, "none"),
    (3, 50, 2, 5, 64, 64, False, False, "none"), (1, 17, 9, 3, 96, 24, False, True, "shared"), (2, 9, 2, 1, 96, 90, False, False, "none"),
    (1, 70, 12, 4, 256, 256, True, True, "shared"), (1, 300, 2, 2, 8, 6, True, True, "heads"), (1, 21, 1, 2, 16, 2, False, True, "shared"),
    (2, 40, 5, 1, 80, 80, False, True, "shared"), (1, 64, 8, 2, 128, 0, False, True, "shared"), (1, 5, 17, 9, 200, 96, False, True, "heads"),
    (1, 1, 32, 8, 128, 128, True, False, "none"), (4, 128, 3, 3, 32, 32, False, True, "shared"), (1, 20, 2, 2, 24, 10, False, False, "none")]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("kind", range(len(KINDS)))
@pytest.mark.parametrize("layout,far,nobody", [("heads", 0, 0.0), ("tokens", 3000, 0.1), ("gaps", 1000000, 0.0)])
def test_forward(dtype, kind, layout, far, nobody):
    b, t, Hq, Hkv, d, r, adjacent, norm, weights = KINDS[kind]
    print(dtype, KINDS[kind], layout, flush=True)
    rot, rows, pos, ws, _ = make(kind, dtype, *KINDS[kind], layout=layout, far=far, nobody=nobody)
    q, k = rows[:, :Hq], rows[:, Hq:]
    wide = torch.full((b, t, Hq + Hkv, d + 8), 5.0, dtype=dtype, device="cuda")
    qo, ko = wide[:, :, :Hq, :d].transpose(1, 2), wide[:, :, Hq:, :d].transpose(1, 2)
    lb.lococo_rows_rotate(rot, q, k, qo, ko, pos)
    assert torch.equal(wide[..., d:], torch.full_like(wide[..., d:], 5.0))
    check_forward(rot, q, ws[0], pos, qo, adjacent, norm, 5.0)
    check_forward(rot, k, ws[1], pos, ko, adjacent, norm, 5.0)
    # either alone, and in place: the same bits
    ko2 = torch.full_like(ko, 5.0)
    lb.lococo_rows_rotate(rot, None, k, None, ko2, pos)
    assert torch.equal(ko2, ko)
    before, real = q.clone(), slice(None) if pos is None else (pos.reshape(b, 1, t, 1) >= 0).expand_as(q)
    lb.lococo_rows_rotate(rot, q, None, q, None, pos)
    assert torch.equal(q[real], qo[real])
    if pos is not None:
        assert torch.equal(q[~real], before[~real])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("pos", [0, 1, 2 ** 24 - 1, 2 ** 24 + 1, 10 ** 8 + 7, 2 ** 31 - 1])
def test_far_positions(dtype, pos):
    """The angle is the exact product: the same rows at one position, whose cosines are known in 64 bits (products of 31 and 24 bits: to 2^-23
    of a turn at the largest)."""
    rot, rows, _, ws, _ = make(3, dtype, 1, 4, 2, 1, 64, 64, False, False, "none", far=0)
    p = torch.full((4,), pos, **I32)
    qo, ko = torch.full_like(rows[:, :2], 5.0), torch.full_like(rows[:, 2:], 5.0)
    lb.lococo_rows_rotate(rot, rows[:, :2], rows[:, 2:], qo, ko, p)
    check_forward(rot, rows[:, :2], None, p, qo, False, False, 5.0)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("size", [0.0, 1e-30, 1e-18, 1e18, 1e25, 1e38])
def test_rows_of_every_size(dtype, size):
    """Squares that leave fp32 on either side; one wild row among tame ones."""
    rot, rows, _, ws, _ = make(5, dtype, 1, 5, 2, 1, 128, 128, False, True, "shared", far=0)
    rows = (rows.float() / rows.float().abs().amax()).to(dtype)
    rows[:, :, 2] = (rows[:, :, 2].float() * size).to(dtype)
    outs = [torch.full_like(rows[:, :2], 5.0), torch.full_like(rows[:, 2:], 5.0)]
    lb.lococo_rows_rotate(rot, rows[:, :2], rows[:, 2:], *outs)
    check_forward(rot, rows[:, :2], ws[0], None, outs[0], False, True, 5.0)
    check_forward(rot, rows[:, 2:], ws[1], None, outs[1], False, True, 5.0)
    if size in (1e18, 1e25):
        gy = [torch.randn(x.shape, device="cuda") for x in outs]
        gx = [torch.empty_like(x) for x in gy]
        lb.lococo_rows_rotate_backward(rot, rows[:, :2], rows[:, 2:], None, *gy, *gx)
        check_backward(rot, rows[:, :2], ws[0], None, gy[0], gx[0], None, False, True)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("odd", [math.nan, math.inf])
def test_a_row_of_nan_stays_by_itself(dtype, odd):
    rot, rows, _, ws, _ = make(6, dtype, 1, 9, 3, 1, 64, 64, False, True, "shared", far=0)
    clean = [torch.empty_like(rows[:, :3]), torch.empty_like(rows[:, 3:])]
    lb.lococo_rows_rotate(rot, rows[:, :3], rows[:, 3:], *clean)
    rows[0, 1, 4, 7] = odd
    outs = [torch.empty_like(x) for x in clean]
    lb.lococo_rows_rotate(rot, rows[:, :3], rows[:, 3:], *outs)
    assert torch.isnan(outs[0][0, 1, 4]).any()
    outs[0][0, 1, 4] = clean[0][0, 1, 4]
    assert torch.equal(outs[0], clean[0]) and torch.equal(outs[1], clean[1])


# ---- the way back
def check_backward(rot, x, w, pos, gy, gx, gw, adjacent, norm, was=0.0):
    b, H, t, d = x.shape
    x, w, gy, gx = x.cpu(), None if w is None else w.cpu(), gy.cpu().double(), gx.cpu().double()
    r, ang = rot.c.rotary_dim, angle_of(rot, pos, b, t)
    real = torch.ones(b, t, dtype=torch.bool) if pos is None else (pos.cpu() >= 0).reshape(b, t)
    gy = gy * real[:, None, :, None]
    want, want_w = ru.backward(x, w, ang, r, adjacent, norm, EPS, gy)
    _, hat, one = ru.normed(x, w, norm, EPS)
    G, W = ru.reach(gy, r, adjacent), ru.weight(w).abs()
    tol = 10 * U * G
    if norm:
        tol = (2 * d + 48) * U * one * (W * G + hat.abs() * (W * G * hat.abs()).mean(-1, keepdim=True))
    bad = ~((gx - want).abs() <= tol + 1e-36)
    assert not bad.any(), (bad.nonzero()[:4].tolist(), ((gx - want).abs() / tol)[bad].max().item())
    assert not gx[~real[:, None, :, None].expand_as(gx)].any()
    if gw is not None:
        dims = (0, 1, 2) if w.dim() == 1 else (0, 2)
        N = b * t * (H if w.dim() == 1 else 1)
        tol = (N + d + 32) * U * ((G * hat.abs()).sum(dims) + abs(was))
        bad = ~((gw.cpu().double() - was - want_w).abs() <= tol + 1e-36)
        assert not bad.any(), bad.nonzero()[:4].tolist()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("kind", range(len(KINDS)))
@pytest.mark.parametrize("layout,far,nobody", [("heads", 0, 0.0), ("tokens", 3000, 0.1)])
def test_backward(dtype, kind, layout, far, nobody):
    b, t, Hq, Hkv, d, r, adjacent, norm, weights = KINDS[kind]
    print(dtype, KINDS[kind], layout, flush=True)
    rot, rows, pos, ws, g = make(kind + 50, dtype, *KINDS[kind], layout=layout, far=far, nobody=nobody)
    q, k = rows[:, :Hq], rows[:, Hq:]
    gy = [torch.randn(x.shape, generator=g).cuda() for x in (q, k)]
    if pos is not None:                                                # what nobody's rows hold may be anything
        for x in gy:
            x[(pos.reshape(b, 1, t, 1) < 0).expand_as(x)] = math.nan
    gx = [torch.full_like(x, math.nan) for x in gy]
    gw = [None if w is None else torch.full(w.shape, 2.0, device="cuda") for w in ws]
    work = lb.rotate_workspace(rot, b * t)
    if work is not None:
        work.fill_(255)
    lb.lococo_rows_rotate_backward(rot, q, k, pos, *gy, *gx, *gw, work)
    for i, x in enumerate((q, k)):
        clean = torch.where(torch.isnan(gy[i]), 0.0, gy[i])
        check_backward(rot, x, ws[i], pos, clean, gx[i], gw[i], adjacent, norm, 2.0)
    # again: the same bits; in place, and either alone
    again = [torch.empty_like(x) for x in gx]
    gw2 = [None if w is None else torch.full(w.shape, 2.0, device="cuda") for w in ws]
    lb.lococo_rows_rotate_backward(rot, q, k, pos, *gy, *again, *gw2, work)
    assert all(torch.equal(x, y) for x, y in zip(gx + [w for w in gw if w is not None], again + [w for w in gw2 if w is not None]))
    own = gy[1].clone()
    lb.lococo_rows_rotate_backward(rot, None, k, pos, None, own, None, own)
    assert torch.equal(own, gx[1])


@pytest.mark.parametrize("weights,hq,hkv", [("shared", 8, 2), ("heads", 3, 3)])
def test_gradient_of_many_rows(weights, hq, hkv):
    """More tiles of positions than workgroups: each takes several in turn."""
    rot, rows, pos, ws, g = make(71, torch.bfloat16, 3, 5001, hq, hkv, 64, 64, False, True, weights, far=100000)
    q, k = rows[:, :hq], rows[:, hq:]
    gy = [torch.randn(x.shape, device="cuda") for x in (q, k)]
    gx = [torch.full_like(x, math.nan) for x in gy]
    gw = [torch.zeros(w.shape, device="cuda") for w in ws]
    lb.lococo_rows_rotate_backward(rot, q, k, pos, *gy, *gx, *gw, lb.rotate_workspace(rot, 3 * 5001))
    for i, x in enumerate((q, k)):
        check_backward(rot, x, ws[i], pos, gy[i], gx[i], gw[i], False, True)


@pytest.mark.parametrize("adjacent,norm,weights", [(False, True, "shared"), (True, True, "heads"), (False, False, "none")])
def test_gradients_against_differences(adjacent, norm, weights):
    """sum(c y) along a direction, by central differences of the 64-bit definition: step 1e-4, error 1e-8 of third derivatives."""
    b, t, Hq, Hkv, d, r = 1, 6, 2, 1, 64, 32
    rot, rows, pos, ws, g = make(81, torch.float32, b, t, Hq, Hkv, d, r, adjacent, norm, weights, far=50)
    q, k = rows[:, :Hq], rows[:, Hq:]
    gy = [torch.randn(x.shape, generator=g).cuda() for x in (q, k)]
    gx = [torch.empty_like(x) for x in gy]
    gw = [None if w is None else torch.zeros(w.shape, device="cuda") for w in ws]
    lb.lococo_rows_rotate_backward(rot, q, k, pos, *gy, *gx, *gw, lb.rotate_workspace(rot, b * t))
    ang = angle_of(rot, pos, b, t)
    for x, w, c, dx, dw in zip((q, k), ws, gy, gx, gw):
        x, c = x.cpu().double(), c.cpu().double()
        v = torch.randn(x.shape, generator=g, dtype=torch.float64)
        f = lambda a, w: (c * ru.forward(a, w, ang, r, adjacent, norm, EPS)).sum().item()
        w = None if w is None else w.cpu().double()
        num = (f(x + 1e-4 * v, w) - f(x - 1e-4 * v, w)) / 2e-4
        assert abs((dx.cpu().double() * v).sum().item() - num) <= 1e-5 * (dx.cpu().double() * v).abs().sum().item()
        if w is not None:
            v = torch.randn(w.shape, generator=g, dtype=torch.float64)
            num = (f(x, w + 1e-4 * v) - f(x, w - 1e-4 * v)) / 2e-4
            assert abs((dw.cpu().double() * v).sum().item() - num) <= 1e-5 * (dw.cpu().double() * v).abs().sum().item()


def test_a_training_step_through_a_scan():
    """Raw rows normed and turned, a scan over them, its backward, and on to the raw rows and the norm's weights: the last step against the
    definition in 64 bits, on the gradients that the scan gave."""
    b, t, H, d, M, B = 1, 48, 2, 64, 16, 16
    rot, rows, _, ws, g = make(91, torch.float32, b, t, H, H, d, d, False, True, "shared", far=0, extra=H)
    q, k, v = rows[:, :H], rows[:, H:2 * H], rows[:, 2 * H:].contiguous()
    qr, kr, o = torch.empty(b, H, t, d, device="cuda"), torch.empty(b, H, t, d, device="cuda"), torch.empty(b, H, t, d, device="cuda")
    cfg = lb.make_config(dtype=torch.float32, batch=b, n_q_heads=H, n_kv_heads=H, head_dim=d, M=M, conv_width=3)
    cw = (torch.randn(M, d, 3, generator=g) * 0.1).cuda()
    lb.lococo_rows_rotate(rot, q, k, qr, kr)
    check_forward(rot, q, ws[0], None, qr, False, True, 0.0)
    lb.lococo_sequence_forward(cfg, qr, kr, v, o, cw, None, lb.Cache(cfg), B, lb.workspace(cfg, t, B))
    d_o = torch.randn(b, H, t, d, generator=g).cuda()
    dq, dk, dv = (torch.empty(b, H, t, d, device="cuda") for _ in range(3))
    dc = [torch.empty(b, H, M, d, device="cuda") for _ in range(2)]
    dcw = torch.zeros_like(cw)
    ws2 = torch.empty(lb.lococo_sequence_backward_workspace_bytes(cfg, t, B), dtype=torch.uint8, device="cuda")
    lb.lococo_sequence_backward(cfg, qr, kr, v, B, cw, None, lb.Cache(cfg), d_o, None, None, dq, dk, dv, *dc, dcw, None, ws2)
    gy = [dq.clone(), dk.clone()]
    gw = [torch.zeros(d, device="cuda") for _ in range(2)]
    lb.lococo_rows_rotate_backward(rot, q, k, None, dq, dk, dq, dk, *gw, lb.rotate_workspace(rot, b * t))
    for x, w, y, dx, dw in zip((q, k), ws, gy, (dq, dk), gw):
        assert y.abs().max() > 0 and torch.isfinite(dx).all()
        check_backward(rot, x, w, None, y, dx, dw, False, True)


def test_captured_and_on_another_stream():
    """Forward and backward in a captured graph, replayed with other rows in between; eager calls on another stream beside it."""
    rot, rows, pos, ws, g = make(95, torch.bfloat16, 2, 100, 4, 2, 128, 128, False, True, "shared", far=9000)
    q, k = rows[:, :4], rows[:, 4:]
    gy = [torch.randn(x.shape, generator=g).cuda() for x in (q, k)]
    outs = [torch.zeros_like(q), torch.zeros_like(k)]
    gx = [torch.zeros_like(x) for x in gy]
    gw = [torch.zeros(128, device="cuda") for _ in range(2)]
    work = lb.rotate_workspace(rot, 200)

    def step(outs, gx, gw, work):
        for x in gw:
            x.zero_()
        lb.lococo_rows_rotate(rot, q, k, *outs, pos)
        lb.lococo_rows_rotate_backward(rot, q, k, pos, *gy, *gx, *gw, work)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(outs, gx, gw, work)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(outs, gx, gw, work)
    for turn in range(4):
        rows.copy_(torch.randn(rows.shape, generator=g).to(rows.dtype))
        pos.copy_(torch.randint(0, 100000, pos.shape, generator=g).int())
        want = [[torch.zeros_like(x) for x in y] for y in (outs, gx, gw)]
        step(*want, torch.empty_like(work))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(outs + gx + gw, sum(want, [])):
            assert torch.equal(a, b), turn


# ---- rows into the pages
def placed(g, b, t, R, spare=2):
    """(slots, pages): every batch entry's rows in pages of its own, in any order"""
    per = -(-(t + R - 1) // R)
    n_pages = b * per + spare
    ids = torch.randperm(n_pages, generator=g)[:b * per].reshape(b, per)
    at = torch.arange(t) + torch.randint(0, R, (b, 1), generator=g)
    return (torch.gather(ids, 1, at // R) * R + at % R).flatten().int(), n_pages


APPENDS = [  # b, t, Hq, Hkv, d, r, adjacent, norm, weights, R
    (32, 1, 32, 8, 128, 128, False, True, "shared", 64), (2, 77, 4, 4, 128, 128, False, False, "none", 16), (1, 130, 6, 2, 64, 32, True, True, "heads", 32),
    (3, 20, 2, 1, 96, 24, False, True, "none", 16), (1, 9, 5, 5, 256, 256, False, True, "shared", 1024), (2, 33, 3, 1, 32, 32, True, False, "none", 16),
    (1, 40, 2, 2, 160, 50, False, True, "shared", 128), (1, 65, 4, 1, 128, 0, False, True, "shared", 64)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("kind", range(len(APPENDS)))
@pytest.mark.parametrize("layout", ["tokens", "heads"])
def test_append(dtype, kind, layout):
    """Codes and scales equal those of the 64-bit definition: every one."""
    b, t, Hq, Hkv, d, r, adjacent, norm, weights, R = APPENDS[kind]
    rot, rows, pos, ws, g = make(kind + 200, dtype, b, t, Hq, Hkv, d, r, adjacent, norm, weights, layout=layout, far=200000, extra=Hkv)
    q, k, v = rows[:, :Hq], rows[:, Hq:Hq + Hkv], rows[:, Hq + Hkv:]
    slots, n_pages = placed(g, b, t, R)
    pages = lb.Pages(dtype=dtype, n_q_heads=Hq, n_kv_heads=Hkv, head_dim=d, page_rows=R, n_pages=n_pages)
    marks = (pages.k_codes, pages.k_scales, pages.v_codes, pages.v_scales)
    for x in marks:
        x.fill_(0x5a)
    pos[::7] = -1                                                      # rows of nobody: with and without a slot
    slots[::14] = -1
    slots[3::29] = n_pages * R
    qo = torch.full((b, Hq, t, d), 5.0, dtype=dtype, device="cuda")
    lb.lococo_pages_append(pages, rot, q, k, v, qo, slots.cuda(), pos)
    check_forward(rot, q, ws[0], pos, qo, adjacent, norm, 5.0)
    ang = ru.angles(pos.cpu(), rot.freqs.cpu()).reshape(b, t, -1) if r else torch.zeros(b, t, 0, dtype=torch.float64)
    keys = ru.forward(k.cpu(), None if ws[1] is None else ws[1].cpu(), ang, r, adjacent, norm, EPS)
    got = [x.cpu() for x in marks]
    want = [torch.full_like(x, 0x5a) for x in got]
    for x, codes, scales in ((keys, *want[:2]), (v.cpu().double(), *want[2:])):
        code, scale = pu.four_bits(x.transpose(1, 2).reshape(b * t, Hkv, d))
        on = (slots >= 0) & (slots < n_pages * R)
        page, row = (slots[on] // R).long(), (slots[on] % R).long()
        code = code[on]
        codes[page, :, row] = code[..., 0::2] | (code[..., 1::2] << 4)
        scales[page, :, :, row] = scale[on]
    for i, (x, y) in enumerate(zip(got, want)):
        assert torch.equal(x, y), (i, (x != y).nonzero()[:4].tolist())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_append_without_a_turn_is_store(dtype):
    """Position 0 and no norm: the rows as they are, ties and all."""
    b, t, H, d, R = 1, 50, 2, 128, 16
    rot, rows, _, ws, g = make(300, dtype, b, t, H, H, d, d, False, False, "none", extra=H)
    rows.copy_((torch.randint(-24, 25, rows.shape, generator=g) * 0.25).to(dtype))      # multiples of a quarter: many ties
    slots, n_pages = placed(g, b, t, R)
    both = [lb.Pages(dtype=dtype, n_q_heads=H, n_kv_heads=H, head_dim=d, page_rows=R, n_pages=n_pages) for _ in range(2)]
    qo = torch.empty(b, H, t, d, dtype=dtype, device="cuda")
    lb.lococo_pages_append(both[0], rot, rows[:, :H], rows[:, H:2 * H], rows[:, 2 * H:], qo, slots.cuda(), torch.zeros(t, **I32))
    lb.lococo_pages_store(both[1], rows[:, H:2 * H], rows[:, 2 * H:], slots.cuda())
    assert torch.equal(qo, rows[:, :H])
    for x, y in zip(arrays_of(both[0]), arrays_of(both[1])):
        assert torch.equal(x, y)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_append_marks_what_is_not_finite(dtype):
    rot, rows, pos, ws, g = make(310, dtype, 1, 20, 2, 2, 64, 64, False, True, "shared", extra=2)
    q, k, v = rows[:, :2], rows[:, 2:4], rows[:, 4:]
    k[0, 0, 3, 5], k[0, 1, 4, 40], v[0, 1, 5, 33] = math.inf, math.nan, -math.inf
    pages = lb.Pages(dtype=dtype, n_q_heads=2, n_kv_heads=2, head_dim=64, page_rows=32, n_pages=1)
    qo = torch.empty_like(q)
    lb.lococo_pages_append(pages, rot, q, k, v, qo, torch.arange(20, **I32), pos)
    assert torch.isfinite(qo.float()).all()
    odd = (pages.k_scales[0] == 255).nonzero().tolist()
    # a norm takes the whole row along
    assert sorted(map(tuple, odd)) == [(0, 0, 3), (0, 1, 3), (1, 0, 4), (1, 1, 4)]
    assert (pages.v_scales[0] == 255).nonzero().tolist() == [[1, 1, 5]]


def test_nothing_to_do_and_refusals():
    rot, rows, pos, ws, g = make(320, torch.bfloat16, 1, 4, 2, 1, 64, 64, False, True, "shared", extra=1)
    q, k, v = rows[:, :2], rows[:, 2:3], rows[:, 3:]
    none = [x[:, :, :0] for x in (q, k)]
    lb.lococo_rows_rotate(rot, *none, *none, torch.empty(0, **I32))
    empty = [torch.empty(x.shape, device="cuda") for x in none]
    gw = [torch.full((64,), 3.0, device="cuda") for _ in range(2)]
    lb.lococo_rows_rotate_backward(rot, *none, None, *empty, *empty, *gw, lb.rotate_workspace(rot, 0))
    assert all((w == 3.0).all() for w in gw)
    qo, ko = torch.empty_like(q), torch.empty_like(k)
    pages = lb.Pages(dtype=torch.bfloat16, n_q_heads=2, n_kv_heads=1, head_dim=64, page_rows=16, n_pages=1)
    slots = torch.arange(4, **I32)
    with pytest.raises(ValueError):
        lb.lococo_rows_rotate(rot, q, k, qo, ko, pos[:3])
    with pytest.raises(ValueError):
        lb.lococo_rows_rotate(rot, q, k, qo, None, pos)
    with pytest.raises(TypeError):
        lb.lococo_rows_rotate(rot, q, k, qo, ko, pos.long())
    with pytest.raises(TypeError):
        lb.lococo_rows_rotate(rot, q, k, qo, ko, pos.cpu())
    with pytest.raises(TypeError):
        lb.lococo_rows_rotate(rot, q, k, qo.float(), ko, pos)
    with pytest.raises(TypeError):
        lb.lococo_pages_append(pages, rot, q, k, v, qo, slots.cpu(), pos)
    with pytest.raises(ValueError):
        lb.lococo_pages_append(pages, rot, q, k, v, qo, slots[:3], pos)
    with pytest.raises(lb.LococoError) as e:
        lb.lococo_rows_rotate(rot, q, k, q[:, :, :1].expand(1, 2, 4, 64).transpose(0, 0), ko, pos)
    assert e.value.status == lb.LOCOCO_EINVAL
    grads = [torch.zeros(x.shape, device="cuda") for x in (q, k, q, k)]
    with pytest.raises(lb.LococoError) as e:
        lb.lococo_rows_rotate_backward(rot, q, k, pos, *grads, torch.zeros(64, device="cuda"))
    assert e.value.status == lb.LOCOCO_EWORKSPACE
    with pytest.raises(TypeError):
        lb.lococo_rows_rotate_backward(rot, q, k, pos, grads[0].bfloat16(), *grads[1:])


def test_another_device_is_refused(monkeypatch):
    """Arrays of a device that is not the current one (here: the only one there is, with another taken for current)."""
    rot, rows, pos, ws, g = make(330, torch.bfloat16, 1, 4, 2, 1, 64, 64, False, True, "shared")
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 1)
    with pytest.raises(TypeError, match="current"):
        lb.lococo_rows_rotate(rot, rows[:, :2], rows[:, 2:], rows[:, :2], rows[:, 2:], pos)
    with pytest.raises(TypeError, match="current"):
        lb.lococo_pages_tree(pos[:2], pos[:1], pos, pos[:, None], pos)
