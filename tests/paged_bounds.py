"""How far a paged decode may be from its definition, with the roundings counted as independent ones, for data where they are.

tests/paged_reference.py bounds every element by the worst case of its sums, which holds for any data and is too wide to notice
operands or weights of 16 bits.  Here each rounding is an error of its own, none larger than its step, and their squares are
added: what the sum of squares predicts is an upper estimate of the size of the whole error (its norm over a result), and eight
times it of any one element (eight deviations)."""
import math

import torch

STEP = 2.0 ** -24  # of fp32, relative


def decode(q, k_rows, v_rows, group):
    """q [heads, d]; k_rows, v_rows [n, kv heads, d]: the visible rows.  Returns (out, deviation before the rounding to the type)."""
    q, k_rows, v_rows = q.double(), k_rows.double(), v_rows.double()
    n, _, d = k_rows.shape
    k, v = (x.repeat_interleave(group, 1).transpose(0, 1) for x in (k_rows, v_rows))   # [heads, n, d]
    s = (k * q[:, None]).sum(-1) / math.sqrt(d)
    w = torch.exp(s - s.amax(1, keepdim=True))
    w = w / w.sum(1, keepdim=True)
    out = (w[..., None] * v).sum(1)
    # A score is a chain of d sums whose partial ones are of the size of the products' norm, or of the score itself: sqrt(d)
    # steps of that, over sqrt(d).  The exponential adds two steps, its argument (difference, scale, product) two of its size.
    size = torch.sqrt(((k * q[:, None]) ** 2).sum(-1) + d * s * s)
    weight = STEP * torch.sqrt(size ** 2 + 4 + 4 * (s - s.amax(1, keepdim=True)) ** 2)
    var = (w[..., None] ** 2 * weight[..., None] ** 2 * (v - out[:, None]) ** 2).sum(1)
    # the weighted sum: a chain of n additions at the most of what has come together; quotient and the pieces' factors
    var = var + STEP ** 2 * (n * (w[..., None] ** 2 * v ** 2).sum(1) + 8 * out ** 2)
    return out, torch.sqrt(var)


def decode_batch(q, k_pages, v_pages, table, keys, group):
    """keys[r]: the rows that request r sees."""
    size = k_pages.shape[1]
    outs, devs = [], []
    for r, at in enumerate(keys):
        at = torch.as_tensor(at, dtype=torch.long)
        if len(at) == 0:
            outs.append(torch.zeros(q.shape[1:], dtype=torch.float64))
            devs.append(torch.zeros(q.shape[1:], dtype=torch.float64))
            continue
        page = torch.as_tensor(table[r], dtype=torch.long)[at // size]
        o, e = decode(q[r], k_pages[page, at % size], v_pages[page, at % size], group)
        outs.append(o)
        devs.append(e)
    return torch.stack(outs), torch.stack(devs)


def rounding(want, dtype):
    """Deviation of one rounding to the type: uniform within half a step at the value's own exponent."""
    return torch.ldexp(torch.full_like(want, torch.finfo(dtype).eps / 2 / math.sqrt(3.0)), torch.frexp(want).exponent - 1)


def excess(got, want, dev, dtype):
    """(norm of the error over the norm that the roundings predict, largest element over its bound); both at most 1 for a result
    whose roundings are those above.  A norm over few elements varies: by less than 8 / sqrt(their number) for uniform errors."""
    err = got.detach().cpu().double() - want
    if dtype == torch.float32:
        norm = torch.sqrt((dev ** 2).sum())                  # rounding to the type is among the steps counted
        bound = 8 * dev + 2 * STEP * want.abs()
    else:
        norm = torch.sqrt((dev ** 2 + rounding(want, dtype) ** 2).sum())
        bound = 8 * dev + torch.finfo(dtype).eps / 2 * want.abs()
    few = 1 + 4 / math.sqrt(want.numel())
    return float(torch.sqrt((err ** 2).sum()) / (few * norm)), float((err.abs() / (bound + 1e-37)).max())
