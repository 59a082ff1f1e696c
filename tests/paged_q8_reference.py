"""Definitions of the paged cache in 8 bits, in 64 bits (torch on the CPU): what codes and scales stand for, the codes and scales of rows, and what an
append leaves behind.  Nothing here is shared with the library."""
import math

import numpy as np
import torch

BLOCK, LEAST, MOST = 16, -117, 120
MOST_VALUE = 1.875 * 2.0 ** 127


def _value(code):
    e, m = (code >> 3) & 15, code & 7
    if e == 15 and m == 7:
        return math.nan
    x = math.ldexp(8 + m, e - 10) if e else math.ldexp(m, -9)
    return -x if code & 128 else x


VALUES = torch.tensor([_value(c) for c in range(256)], dtype=torch.float64)


def values(codes, scale):
    """codes uint8 [pages, size, heads, d], scale uint8 [pages, heads, size / 16] -> what they are worth, [pages, size, heads, d]."""
    factor = torch.ldexp(torch.ones((), dtype=torch.float64), scale.int() - 127)
    return VALUES[codes.long()] * factor.repeat_interleave(BLOCK, 2).transpose(1, 2)[..., None]


def round_code(y):
    """The code nearest to each y (in units of the scale), ties to the even mantissa; NaN for what is not finite."""
    a = y.abs()
    e = torch.frexp(a).exponent - 1
    step = torch.ldexp(torch.ones_like(a), torch.clamp(e, min=-6) - 3)
    n = a / step                                   # exact: a power of two
    whole = torch.floor(n)
    rest = n - whole
    up = (rest > 0.5) | ((rest == 0.5) & (whole % 2 == 1))
    r = (whole + up) * step
    table = VALUES[:127]
    code = torch.searchsorted(table, r.contiguous()).clamp(max=126)
    assert bool((table[code] == r)[torch.isfinite(y) & (a <= 448)].all())
    code = code + 128 * torch.signbit(y).long()
    return torch.where(torch.isfinite(y), code, 127).to(torch.uint8)


def exponent(top):
    """The smallest e with top <= 448 * 2^e, within its limits."""
    m, e = torch.frexp(top.double())
    need = torch.where(m > 0.875, e - 8, e - 9)
    return torch.where(top > 0, need, LEAST).clamp(LEAST, MOST)


def finite_top(x, dims):
    return torch.where(torch.isfinite(x), x.abs(), 0.0).amax(dims)


def scaled(x, e):
    """x in units of 2^e, at most what fp32 has."""
    y = torch.where(torch.isfinite(x), x.clamp(-MOST_VALUE, MOST_VALUE), x)
    return torch.ldexp(y, -e)


def groups(slots):
    """(block, [(token, row)]) of the blocks of 16 rows that a call writes, by the slots of its tokens."""
    out = {}
    for t, s in enumerate(slots):
        if s >= 0:
            out.setdefault(int(s) // BLOCK, []).append((t, int(s) % BLOCK))
    return out


def check_append(got_codes, got_scale, codes, scale, x, err, slots, what):
    """One side of the pool after an append, against the rows x [tokens, heads, d] in 64 bits, known up to err (a tensor, or 0: then
    scales and codes have one right answer).  codes, scale: the pool before."""
    n_pages, size = codes.shape[:2]
    want_codes, want_scale, free = codes.clone(), scale.clone(), torch.zeros(codes.shape, dtype=torch.bool)
    for block, rows in groups(slots).items():
        p, b = divmod(block, size // BLOCK)
        if p >= n_pages:
            continue
        at = torch.tensor([t for t, _ in rows])
        row = torch.tensor([r for _, r in rows])
        xs = x[at]
        anew = bool((row == 0).any())
        old = scale[p, :, b].int() - 127
        tops = []
        for sign in (-1.0, 1.0):
            es = err[at] if torch.is_tensor(err) else 0.0
            tops.append(exponent((finite_top(xs.abs() + sign * es, (0, 2))).clamp(min=0)))
        low, high = tops
        if not anew:
            low, high = torch.maximum(low, old), torch.maximum(high, old)
        e = got_scale[p, :, b].int() - 127
        assert bool(((e >= low) & (e <= high)).all()), (what, "scale of block", block, e.tolist(), low.tolist(), high.tolist())
        want_scale[p, :, b] = got_scale[p, :, b]
        span = slice(b * BLOCK, (b + 1) * BLOCK)
        if not anew:
            grown = (e > old)[None, :, None]
            again = round_code(torch.ldexp(VALUES[codes[p, span].long()], (old - e)[None, :, None]))
            want_codes[p, span] = torch.where(grown, again, codes[p, span])
        y = scaled(xs, e[None, :, None])
        if not torch.is_tensor(err):
            want_codes[p, b * BLOCK + row] = round_code(y)
        else:
            free[p, b * BLOCK + row] = True
            got = VALUES[got_codes[p, b * BLOCK + row].long()]
            ulp = torch.ldexp(torch.ones_like(y), torch.clamp(torch.frexp(y.abs()).exponent - 1, min=-6) - 3)
            bound = ulp / 2 + torch.ldexp(err[at], -e[None, :, None])
            ok = torch.where(torch.isfinite(xs), (got - y).abs() <= bound, torch.isnan(got))
            assert bool(ok.all()), (what, "codes of block", block, int((~ok).sum()), (~ok).nonzero()[0].tolist())
    isnan = (want_codes & 127) == 127
    same = (got_codes == want_codes) | (isnan & ((got_codes & 127) == 127)) | free
    assert bool(same.all()), (what, "codes", int((~same).sum()), (~same).nonzero()[:4].tolist())
    assert torch.equal(got_scale, want_scale), (what, "scales", (got_scale != want_scale).nonzero()[:4].tolist())


def random_pool(n_pages, size, heads, d, seed, spread=1):
    """Codes of normal values with their blocks' scales, uint8 on the CPU."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(n_pages, size // BLOCK, BLOCK, heads, d, generator=g, dtype=torch.float64)
    x = x * torch.ldexp(torch.ones((), dtype=torch.float64), torch.randint(-spread, spread + 1, (n_pages, size // BLOCK, 1, heads, 1), generator=g))
    e = exponent(x.abs().amax((2, 4)))
    codes = round_code(torch.ldexp(x, -e[:, :, None, :, None])).reshape(n_pages, size, heads, d)
    return codes, (e + 127).to(torch.uint8).transpose(1, 2).contiguous()


def device_codes(codes, order):
    """The pool on the GPU, in one of several layouts."""
    n, size, heads, d = codes.shape
    if order == "rows":
        t = torch.empty(n, size, heads, d, dtype=torch.uint8, device="cuda")
    elif order == "heads":
        t = torch.empty(n, heads, size, d, dtype=torch.uint8, device="cuda").transpose(1, 2)
    else:  # "wide": rows of a wider allocation, pages with room between them
        t = torch.empty(n, size + 3, heads, d + 32, dtype=torch.uint8, device="cuda")[:, :size, :, 16:16 + d]
    return t.copy_(codes)


def tokens_of(rng, n_req, size, cached_hi, new_lo, new_hi, pad, spare=2):
    """Slots of the new tokens of a batch, and the number of pages."""
    cached, new = rng.integers(0, cached_hi + 1, n_req), rng.integers(new_lo, new_hi + 1, n_req)
    need = -(-(cached + new) // size)
    pool, at, slots = rng.permutation(int(need.sum()) + spare), 0, []
    for r in range(n_req):
        row = cached[r] + np.arange(new[r])
        slots.append(pool[at + row // size] * size + row % size)
        at += int(need[r])
    return np.concatenate(slots + [np.full(pad, -1)]).astype(np.int64), len(pool)
