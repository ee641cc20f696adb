"""Plain implementations, in 64 bits on the CPU and written from lococo.h's definitions, of norm and rotation of rows, of the numbers of turns
with drafted trees, and of attention under masks."""
import math

import torch

import pages_util as pu


def pairs(r, adjacent):
    """[(a, b)] of the r / 2 pairs of channels"""
    return [(2 * i, 2 * i + 1) if adjacent else (i, i + r // 2) for i in range(r // 2)]


def angles(positions, freqs):
    """[rows, r / 2]: whole numbers times fp32 frequencies, exact in 64 bits up to 2^29"""
    return positions.double()[:, None] * freqs.double()[None]


def normed(x, w, norm, eps):
    """(n, x over its root mean square, one over that root) of rows [b, heads, t, d]; w None, [d] or [heads, d]"""
    x = x.double()
    one = 1.0 / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) if norm else torch.ones_like(x[..., :1])
    hat = x * one
    return hat * weight(w), hat, one


def weight(w):
    if w is None:
        return torch.ones((), dtype=torch.float64)
    return w.double() if w.dim() == 1 else w.double()[:, None, :]


def turn(n, angle, r, adjacent, back=False):
    """rows [b, heads, t, d] turned by angle [b, t, r / 2], or the other way"""
    y, c, s = n.clone(), torch.cos(angle)[:, None], torch.sin(angle)[:, None] * (-1.0 if back else 1.0)
    if r:
        a, b = (torch.tensor(i) for i in zip(*pairs(r, adjacent)))
        y[..., a], y[..., b] = n[..., a] * c - n[..., b] * s, n[..., b] * c + n[..., a] * s
    return y


def reach(n, r, adjacent):
    """|n_a| + |n_b| for either channel of a pair, |n| for channels that are not turned: what a turned value's error is measured by"""
    n = n.abs()
    y = n.clone()
    if r:
        a, b = (torch.tensor(i) for i in zip(*pairs(r, adjacent)))
        y[..., a] = y[..., b] = n[..., a] + n[..., b]
    return y


def forward(x, w, angle, r, adjacent, norm, eps):
    return turn(normed(x, w, norm, eps)[0], angle, r, adjacent)


def backward(x, w, angle, r, adjacent, norm, eps, gy):
    """(d_x, d_w) by the formula in lococo.h's terms; d_w as w lies (None without weights)"""
    _, hat, one = normed(x, w, norm, eps)
    gn = turn(gy.double(), angle, r, adjacent, back=True)
    gw = None if w is None else (gn * hat).sum((0, 1, 2)) if w.dim() == 1 else (gn * hat).sum((0, 2))
    if not norm:
        return gn, None
    g = gn * weight(w)
    return one * (g - hat * (g * hat).mean(-1, keepdim=True)), gw


def tree(starts, held, parents, words, tokens, bases=None):
    """(masks [tokens][words] as whole numbers below 2^32, positions) row by row"""
    masks, positions = [[0] * words for _ in range(tokens)], [-1] * tokens
    for i in range(len(held)):
        a, b = starts[i], starts[i + 1]
        base = bases[i] if bases is not None else max(held[i], 0) - (b - a)
        for x in range(min(b - a, 32 * words)):
            seen, up = [], x
            while up >= 0:
                seen.append(up)
                p = parents[a + up]
                up = p if 0 <= p < up else -1
            for j in seen:
                masks[a + x][j // 32] |= 1 << (j % 32)
            positions[a + x] = base + len(seen) - 1 if base >= 0 else -1
    return masks, positions


def keep(n_pages, page_rows, tables, starts, held, slots, kept, ring, ends):
    """lococo_pages_keep, request by request; a dict of lists"""
    R, width = page_rows, len(tables[0])
    tokens = len(slots)
    ring, after, back, rows = list(ring), [], [], 0
    sources, targets = [-1] * tokens, [-1] * tokens
    for i, h in enumerate(held):
        a, b = starts[i], starts[i + 1]
        h = max(0, min(h, width * R))
        if b == a or b - a > h or slots[a] < 0:
            after.append(h)
            continue
        to = a
        for x in range(a, b):
            if kept[x]:
                if to != x:
                    sources[x], targets[x] = slots[x], slots[to]
                to += 1
        rows += to - a
        after.append(h - (b - to))
        back += tables[i][-(-after[-1] // R):-(-h // R)]
    for j, p in enumerate(back):
        ring[(ends[1] + j) % n_pages] = p
    return dict(held=after, ends=[ends[0], ends[1] + len(back)], sources=sources, targets=targets, totals=[rows, len(back)], ring=ring)


def attention(q, tables, starts, held, masks, arrays, page_rows, group, scale):
    """pages_util.attention with what a new row sees named by masks [tokens][words] (whole numbers below 2^32)"""
    kc, ks, vc, vs = arrays
    n_pages = kc.shape[0]
    H, T, d = q.shape
    o, mass, size = torch.full((H, T, d), math.nan, dtype=torch.float64), torch.zeros(H, T, d, dtype=torch.float64), torch.zeros(H, T, dtype=torch.float64)
    for i in range(len(held)):
        t0, t1 = starts[i], starts[i + 1]
        n, w = max(0, min(held[i], tables.shape[1] * page_rows)), t1 - t0
        rows = [(int(tables[i, j // page_rows]), j % page_rows) for j in range(n)]
        there = torch.tensor([0 <= p < n_pages for p, _ in rows], dtype=torch.bool)
        pi = torch.tensor([p if 0 <= p < n_pages else 0 for p, _ in rows], dtype=torch.long)
        ri = torch.tensor([r for _, r in rows], dtype=torch.long)
        for h in range(H // group):
            k = pu.values(pu.unpack(kc[pi, h, ri]), ks[pi, h, :, ri]) if n else torch.zeros(0, d, dtype=torch.float64)
            v = pu.values(pu.unpack(vc[pi, h, ri]), vs[pi, h, :, ri]) if n else torch.zeros(0, d, dtype=torch.float64)
            for t in range(t0, t1):
                bits = masks[t]
                named = [j < n - w or (j - (n - w) < 32 * len(bits) and bits[(j - (n - w)) // 32] >> ((j - (n - w)) % 32) & 1) for j in range(n)]
                see = there & torch.tensor(named, dtype=torch.bool)
                for a in range(h * group, (h + 1) * group):
                    if not see.any():
                        o[a, t] = 0.0
                        continue
                    x = q[a, t].double()
                    p = torch.softmax((k[see] @ x) * scale, 0)
                    o[a, t] = p @ v[see]
                    mass[a, t] = p @ v[see].abs()
                    size[a, t] = (k[see].abs() @ x.abs()).max() * scale
    return o, mass, size
