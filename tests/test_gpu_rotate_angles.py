"""Angles of rotated rows at any position, against whole-number arithmetic: products of 31-bit positions and 24-bit frequencies have more bits
than a number of 64 bits holds, and so has what is left of them without their whole turns.

Rows (1, 0) in every pair give the cosine and the sine themselves: no norm, no weights, both products exact."""
import math
from fractions import Fraction

import pytest
import torch

import pages_util as pu
import rotate_util as ru
from paper_2406_05317_amd import binding as lb
from test_gpu_pages import arrays_of

pytestmark = pytest.mark.gpu
I32 = dict(dtype=torch.int32, device="cuda")
U = 2.0 ** -24
TWO_PI = 2 * Fraction("3.14159265358979323846264338327950288419716939937510582097494459230781640628620899862803482534211706798")


def left_over(positions, freqs):
    """[rows, pairs]: the exact products without their whole turns, in [-pi, pi], rounded once to 64 bits"""
    f = [Fraction(x) for x in freqs.tolist()]
    out = []
    for p in positions.tolist():
        turns = [p * x / TWO_PI for x in f]
        out.append([float((t - round(t)) * TWO_PI) for t in turns])
    return torch.tensor(out, dtype=torch.float64)


def far(seed, n, pairs, least=0, low=-4):
    """Positions of every size from 2^least up to the largest, frequencies from 10^low to 10^4 radians a position."""
    g = torch.Generator().manual_seed(seed)
    pos = (2.0 ** (least + (31 - least) * torch.rand(n, generator=g, dtype=torch.float64))).long() - 1
    pos[:4] = torch.tensor([2 ** 31 - 1, 2 ** 30 + 12345, 2 ** 29 + 1, 2 ** 29 - 1])
    freqs = (10.0 ** (low + (4 - low) * torch.rand(pairs, generator=g, dtype=torch.float64))).float()
    return pos.int(), freqs


@pytest.mark.parametrize("adjacent", [False, True])
def test_cosines_and_sines_of_far_positions(adjacent):
    """8 u: the half turns left over are rounded to fp32 (pi 2^-25 < 1.6 u at most), the function's own error is some units."""
    n, d = 200, 128
    pos, freqs = far(1, n, d // 2)
    rot = lb.Rotation(dtype=torch.float32, n_q_heads=1, n_kv_heads=1, head_dim=d, freqs=freqs.cuda(), adjacent=adjacent)
    a, b = (torch.tensor(i) for i in zip(*ru.pairs(d, adjacent)))
    x = torch.zeros(1, 1, n, d)
    x[..., a] = 1.0
    out = torch.empty(1, 1, n, d, device="cuda")
    lb.lococo_rows_rotate(rot, x.cuda(), None, out, None, pos.cuda())
    got, angle = out.cpu().double()[0, 0], left_over(pos, freqs)
    for want, mine in ((torch.cos(angle), got[:, a]), (torch.sin(angle), got[:, b])):
        bad = ~((mine - want).abs() <= 8 * U)
        assert not bad.any(), (bad.sum().item(), (mine - want).abs().max().item() / U)


@pytest.mark.parametrize("top", [100, 4096, 2 ** 31 - 1])
def test_cosines_and_sines_to_steps_of_their_own_size(top):
    """Relative to each value, those beside a zero among them.  The angle is counted from the nearest quarter turn, at most 1/4 of a half turn: its
    rounding, u of it, moves the sine by at most u of the sine and the cosine by pi/4 tan(pi/4) u < u of the cosine.  The function's own error: 2
    steps, 4 u where a step is largest.  One u more for the angle's 2^-52 in 64 bits: no value here is below 2^-20."""
    n, d = 400, 128
    g = torch.Generator().manual_seed(top % 1000)
    pos = (torch.rand(n, generator=g, dtype=torch.float64) * top).long().int()
    freqs = (10000.0 ** (-torch.arange(0, d, 2, dtype=torch.float64) / d)).float()
    out = torch.empty(2, 1, 1, n, d, device="cuda")
    rot = lb.Rotation(dtype=torch.float32, n_q_heads=1, n_kv_heads=1, head_dim=d, freqs=freqs.cuda())
    x = torch.zeros(1, 1, n, d, device="cuda")
    x[..., :d // 2] = 1.0
    lb.lococo_rows_rotate(rot, x, None, out[0], None, pos.cuda())
    v = torch.zeros_like(x)
    pages = lb.Pages(dtype=torch.float32, n_q_heads=1, n_kv_heads=1, head_dim=d, page_rows=16, n_pages=n // 16)
    lb.lococo_pages_append(pages, rot, x, v, v, out[1], torch.arange(n, **I32), pos.cuda())
    angle = left_over(pos, freqs)
    want = torch.cat((torch.cos(angle), torch.sin(angle)), -1)
    live = want.abs() >= 2.0 ** -20
    for got in out.cpu().double()[:, 0, 0]:
        bad = live & ~((got - want).abs() <= 6 * U * want.abs())
        assert not bad.any(), (bad.sum().item(), ((got - want).abs() / want.abs())[bad].max().item() / U)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("adjacent", [False, True])
@pytest.mark.parametrize("least,low", [(0, -4), (30, 3)])
def test_codes_of_far_positions(dtype, adjacent, least, low):
    """Codes and scales of appended keys are those of the exact angles, every one (values of 64 bits: one in 10^10 lies where two exact
    computations could take neighbours).  Rounded products of the largest positions, off by up to 2^-9, get some of 65536 wrong."""
    n, H, d, R = 256, 2, 128, 32
    pos, freqs = far(2, n, d // 2, least, low)
    g = torch.Generator().manual_seed(3)
    rows = torch.randn(1, 3 * H, n, d, generator=g).to(dtype).cuda()
    rot = lb.Rotation(dtype=dtype, n_q_heads=H, n_kv_heads=H, head_dim=d, freqs=freqs.cuda(), adjacent=adjacent)
    pages = lb.Pages(dtype=dtype, n_q_heads=H, n_kv_heads=H, head_dim=d, page_rows=R, n_pages=n // R)
    qo = torch.empty(1, H, n, d, dtype=dtype, device="cuda")
    lb.lococo_pages_append(pages, rot, rows[:, :H], rows[:, H:2 * H], rows[:, 2 * H:], qo, torch.arange(n, **I32), pos.cuda())
    keys = ru.turn(rows[:, H:2 * H].cpu().double(), left_over(pos, freqs)[None], d, adjacent)
    code, scale = pu.four_bits(keys[0].transpose(0, 1))
    got = arrays_of(pages)
    want = torch.zeros_like(got[0]), torch.zeros_like(got[1])
    page, row = torch.arange(n) // R, torch.arange(n) % R
    want[0][page, :, row] = code[..., 0::2] | (code[..., 1::2] << 4)
    want[1][page, :, :, row] = scale
    for i in range(2):
        assert torch.equal(got[i].cpu(), want[i]), (i, (got[i].cpu() != want[i]).sum().item())
    turned = ru.turn(rows[:, :H].cpu().double(), left_over(pos, freqs)[None], d, adjacent)
    tol = 16 * U * ru.reach(rows[:, :H].cpu().double(), d, adjacent) + (2.0 ** -8 * turned.abs() if dtype == torch.bfloat16 else 0.0)
    assert ((qo.cpu().double() - turned).abs() <= tol).all()
