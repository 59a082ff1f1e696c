"""Definitions of the paged cache's operators in 64 bits (numpy / torch on the CPU), and bounds on what rounding may do.

Nothing here is shared with the library: lists and loops where that says most plainly what is meant."""
import math

import numpy as np
import torch

INT_MAX = 2 ** 31 - 1


def page_map(cached, new, first, page, free, table, n_slots):
    """What tr_page_map leaves behind: table, kv_lens, cu, slots, pos, counts as Python integers in int64 arrays."""
    table = np.array(table, dtype=np.int64).copy()
    blocks = table.shape[1]
    cached, new = [max(int(x), 0) for x in cached], [max(int(x), 0) for x in new]
    slots, pos = np.full(n_slots, -1, np.int64), np.zeros(n_slots, np.int64)
    cu, used, at, lens = [0], 0, 0, []
    for r, (c, f) in enumerate(zip(cached, new)):
        have, need = -(-c // page), -(-(c + f) // page)
        ids = {}
        for b in range(have, min(need, have + len(free) + blocks + n_slots)):   # behind that nothing is looked at
            ids[b] = int(free[used + b - have]) if used + b - have < len(free) else -1
            if b < blocks:
                table[r, b] = ids[b]
        used += need - have
        for i in range(min(f, max(n_slots - at, 0))):
            b, row = divmod(c + i, page)
            pid = -1 if b >= blocks else int(table[r, b]) if b < have else ids[b]
            slot = pid * page + row
            slots[at + i] = slot if pid >= 0 and slot <= INT_MAX else -1
            p = (c if first is None else int(first[r])) + i
            pos[at + i] = (p + 2 ** 31) % 2 ** 32 - 2 ** 31
        at += f
        cu.append(min(at, INT_MAX))
        lens.append(min(c + f, INT_MAX))
    return table, np.array(lens, np.int64), np.array(cu, np.int64), slots, pos, np.array([min(at, INT_MAX), min(used, INT_MAX)])


def frequencies(rot, base, scaling="none", factor=1.0, original=0.0, slow=1.0, fast=32.0):
    out = []
    for m in range(rot // 2):
        theta = base ** (-2.0 * m / rot)
        if scaling == "linear":
            theta /= factor
        elif scaling == "base":
            theta = (base * factor ** (rot / (rot - 2.0))) ** (-2.0 * m / rot)
        elif scaling == "parts":
            turns = original * theta / (2.0 * math.pi)
            keep = min(max((turns - slow) / (fast - slow), 0.0), 1.0)
            theta = keep * theta + (1.0 - keep) * theta / factor
        out.append(theta)
    return np.array(out)


def heads(x, weight, eps, pos, freq, layout, amplitude=1.0):
    """Norm, then rotation, of x [tokens, heads, d].  Returns (values, size): size is the sum of the magnitudes of what a
    result is put together from, before amplitude."""
    x = x.double()
    d, half = x.shape[-1], len(freq)
    if weight is not None:
        x = x / torch.sqrt((x * x).sum(-1, keepdim=True) / d + eps) * weight.double()
    y, size = x.clone(), x.abs()
    if half:
        angle = pos.double()[:, None] * torch.from_numpy(np.asarray(freq, np.float64))
        c, s = torch.cos(angle)[:, None], torch.sin(angle)[:, None]
        one = torch.arange(half) if layout == 1 else 2 * torch.arange(half)
        two = one + half if layout == 1 else one + 1
        a, b = x[..., one], x[..., two]
        y[..., one], y[..., two] = amplitude * (a * c - b * s), amplitude * (b * c + a * s)
        both = abs(amplitude) * (a.abs() + b.abs())
        size = size.clone()
        size[..., one], size[..., two] = both, both
    return y, size


def heads_bound(want, size, dtype):
    """Half a step of the type, and the fp32 steps before it, each 2^-24 of `size`: the sum of squares (8 products in a row and up
    to 5 additions over the lanes), mean, eps, root and quotient (3), both factors (2), cosine and sine and their amplitude (3),
    two products and their sum (3): 25, of which those of the norm reach a result once for either of its two terms."""
    return torch.finfo(dtype).eps / 2 * want.abs() + 26 * 2.0 ** -24 * size + 1e-37


def visible(length, window, sinks):
    return [j for j in range(length) if window == 0 or j >= length - window or j < sinks]


def decode(q, k_rows, v_rows, keys, group):
    """q [heads, d]; k_rows, v_rows [n, kv heads, d] the visible rows; returns (out, bound before the rounding to the type)."""
    hq, d = q.shape
    out, bound = torch.zeros(hq, d, dtype=torch.float64), torch.zeros(hq, d, dtype=torch.float64)
    n = len(keys)
    if n == 0:
        return out, bound
    q, k_rows, v_rows = q.double(), k_rows.double(), v_rows.double()
    for h in range(hq):
        k, v = k_rows[:, h // group], v_rows[:, h // group]
        s = k @ q[h] / math.sqrt(d)
        w = torch.exp(s - s.max())
        w = w / w.sum()
        out[h] = w @ v
        # a score is a sum of d products in fp32: off by at most (d + 2) steps of the sum of magnitudes; a weight by that, by the
        # exponential (scaled score and exponent: 2^-20) and by its split into two bf16 parts (2^-16); numerator and
        # denominator each; sums run in chains of at most n / 16 additions and 64 more inside a step and over the pieces
        score = (d + 2) * 2.0 ** -24 * float((k.abs() @ q[h].abs()).max()) / math.sqrt(d)
        bound[h] = (2 * (score + 2.0 ** -20 + 2.0 ** -16) + 2 * (n / 16 + 64) * 2.0 ** -24) * (w @ v.abs())
    return out, bound


def decode_batch(q, k_pages, v_pages, table, lens, window, sinks, group, n_pages=None):
    """k_pages, v_pages [pages, size, kv heads, d] on the CPU.  Keys of pages outside the pool have no weight."""
    n_pages = k_pages.shape[0] if n_pages is None else n_pages
    size = k_pages.shape[1]
    outs, bounds = [], []
    for r in range(q.shape[0]):
        length = min(max(int(lens[r]), 0), table.shape[1] * size)
        keys = [j for j in visible(length, window, sinks) if 0 <= int(table[r, j // size]) < n_pages]
        at = torch.tensor(keys, dtype=torch.long)
        page = table[r].long()[at // size] if keys else at
        o, b = decode(q[r], k_pages[page, at % size], v_pages[page, at % size], keys, group)
        outs.append(o)
        bounds.append(b)
    return torch.stack(outs), torch.stack(bounds)


def assert_within(got, want, bound, what):
    got = got.detach().cpu().double()
    bad = ~((got - want).abs() <= bound)
    assert not bool(bad.any()), "%s: %d of %d outside the bound, worst %.3g of it, at %s" % (
        what, int(bad.sum()), bad.numel(), float(((got - want).abs() / bound.clamp(min=1e-300))[bad].max()), bad.nonzero()[0].tolist())
