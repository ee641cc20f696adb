"""Plain implementations of the operators on paged 4-bit rows, in 64 bits on the CPU, written from lococo.h's definitions."""
import math

import torch

MAGNITUDES = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


def four_bits(x):
    """(codes 0 .. 15, scale bytes) of rows [.., d]."""
    y = x.double().unflatten(-1, (-1, 32))
    a = y.abs().amax(-1)
    odd = ~torch.isfinite(y).all(-1)
    a = torch.where(odd, 1.0, a)
    e = torch.full(a.shape, -100, dtype=torch.int64)
    for n in range(-98, 129):                                   # the definition, exponent by exponent
        p = 2.0 ** n
        here = (a >= p) & (a < 2 * p)
        e = torch.where(here, torch.clamp(torch.tensor(n - 2) + (a > 1.75 * p).long(), -100, 125), e)
    z = y.abs() / (2.0 ** e.double())[..., None]
    grid = torch.tensor(MAGNITUDES, dtype=torch.float64)
    dist = (z[..., None] - grid).abs()
    dist[..., 1::2] += 1e-9                                     # ties to the even code (distances are multiples of 2^-24 apart, or equal)
    code = dist.argmin(-1) | ((torch.signbit(y)).long() << 3)
    code = torch.where(odd[..., None], 0, code)
    return code.flatten(-2).to(torch.uint8), torch.where(odd, 255, e + 127).to(torch.uint8)


def values(code, scale):
    """64-bit values of codes [.., d] and scale bytes [.., d / 32]."""
    c = code.long()
    v = torch.tensor(MAGNITUDES, dtype=torch.float64)[c & 7] * torch.where(c >= 8, -1.0, 1.0)
    s = torch.where(scale == 255, math.nan, 2.0 ** (scale.double() - 127))
    return (v.unflatten(-1, (-1, 32)) * s[..., None]).flatten(-2)


def unpack(byte):
    return torch.stack((byte & 15, byte >> 4), -1).flatten(-2)


def page_values(codes, scales, page, head, row):
    """[d] of one row out of the arrays of the pages (CPU copies)."""
    return values(unpack(codes[page, head, row]), scales[page, head, :, row])


def attention(q, tables, starts, held, arrays, page_rows, group, scale):
    """(o, sum of p |v|, the most sum |q k| scale of a query) for q [heads, tokens, d]; NaN where the definition gives NaN."""
    kc, ks, vc, vs = arrays
    n_pages = kc.shape[0]
    H, T, d = q.shape
    o, mass, size = torch.full((H, T, d), math.nan, dtype=torch.float64), torch.zeros(H, T, d, dtype=torch.float64), torch.zeros(H, T, dtype=torch.float64)
    for i in range(len(held)):
        t0, t1 = starts[i], starts[i + 1]
        n = max(0, min(held[i], tables.shape[1] * page_rows))
        rows = [(int(tables[i, j // page_rows]), j % page_rows) for j in range(n)]
        there = torch.tensor([0 <= p < n_pages for p, _ in rows], dtype=torch.bool)
        pi = torch.tensor([p if 0 <= p < n_pages else 0 for p, _ in rows], dtype=torch.long)
        ri = torch.tensor([r for _, r in rows], dtype=torch.long)
        for h in range(H // group):
            k = values(unpack(kc[pi, h, ri]), ks[pi, h, :, ri]) if n else torch.zeros(0, d, dtype=torch.float64)
            v = values(unpack(vc[pi, h, ri]), vs[pi, h, :, ri]) if n else torch.zeros(0, d, dtype=torch.float64)
            for t in range(t0, t1):
                see = there & (torch.arange(n) <= n - (t1 - t))
                for a in range(h * group, (h + 1) * group):
                    if not see.any():
                        o[a, t] = 0.0
                        continue
                    x = q[a, t].double()
                    s = (k[see] @ x) * scale
                    p = torch.softmax(s, 0)
                    o[a, t] = p @ v[see]
                    mass[a, t] = p @ v[see].abs()
                    size[a, t] = (k[see].abs() @ x.abs()).max() * scale
    return o, mass, size


def plan(n_pages, page_rows, tokens, new, held, tables, ring, ends):
    """The plan of lococo.h, request by request; returns a dict of lists (tables and ring as they are afterwards)."""
    P, R, width = n_pages, page_rows, len(tables[0])
    tables, ring = [list(r) for r in tables], list(ring)
    before = list(ring)
    head, tail = ends
    avail = max(0, min(tail - head, P))
    slots, positions = [-1] * tokens, [-1] * tokens
    starts, after, back = [], [], []
    at = asked = taken = laid = refused = 0
    for i, (w, h) in enumerate(zip(new, held)):
        h = max(0, min(h, width * R))
        starts.append(min(at, tokens))
        have = -(-h // R)
        if w < 0:
            back += tables[i][:have]
            after.append(0)
            continue
        want = -(-(h + w) // R) - have
        fits = at + w <= tokens and have + want <= width
        need = want if fits else 0
        good = fits and (need == 0 or asked + need <= avail)
        if good:
            for j in range(need):
                tables[i][have + j] = before[(head + asked + j) % P]
            for x in range(w):
                page = tables[i][(h + x) // R]
                slots[at + x] = page * R + (h + x) % R if 0 <= page < P else -1
                positions[at + x] = h + x
            taken, laid = taken + need, laid + w
        else:
            refused += 1
        after.append(h + w if good else h)
        asked += need
        at += w
    starts.append(min(at, tokens))
    for j, p in enumerate(back):
        ring[(tail + j) % P] = p
    return dict(held=after, ends=[head + taken, tail + len(back)], starts=starts, slots=slots, positions=positions,
                totals=[laid, taken, len(back), refused], tables=tables, ring=ring)
