"""The bounds of tests/paged_bounds.py notice what they are for: decodes in fp32, on the CPU, in which operands or weights keep
fewer bits than the call promises lie outside them, and one that keeps all of them lies inside."""
import math

import pytest
import torch

from tests import paged_bounds as P


def few_bits(x, bits):
    m, e = torch.frexp(x.double())
    return torch.ldexp(torch.round(m * 2.0 ** bits) / 2.0 ** bits, e).float()


def bf16(x):
    return x.to(torch.bfloat16).float()


def in_fp32(q, k, v, group, mistake):
    """One addition after another, as unkind an order as there is."""
    q, k, v = q.float(), k.float(), v.float()
    if mistake == "scores":
        q, k = few_bits(q, 16), few_bits(k, 16)
    if mistake == "values":
        v = few_bits(v, 16)
    k, v = (x.repeat_interleave(group, 1).transpose(0, 1) for x in (k, v))
    s = torch.zeros(k.shape[:2])
    for i in range(k.shape[2]):
        s = s + k[..., i] * q[:, None, i]
    w = torch.exp2((s - s.amax(1, keepdim=True)) * torch.tensor(math.log2(math.e) / math.sqrt(k.shape[2])).float())
    total = w.sum(1, keepdim=True)
    if mistake == "weights":
        w = few_bits(w, 16)
    if mistake == "two parts":
        w = bf16(w) + bf16(w - bf16(w))
    if mistake == "half":
        w = w.half().float()
    if mistake == "one part":
        w = bf16(w)
    o = torch.zeros(k.shape[0], k.shape[2])
    for j in range(k.shape[1]):
        o = o + w[:, j, None] * v[:, j]
    return o / total


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n", [7, 60, 513])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_bounds_hold_and_notice(dtype, n, d):
    g = torch.Generator().manual_seed(n + d)
    q = (torch.randn(16, d, generator=g) * 0.5).to(dtype)
    k, v = (torch.randn(n, 4, d, generator=g).to(dtype) for _ in range(2))
    want, dev = P.decode(q, k, v, 4)
    norm, element = P.excess(in_fp32(q, k, v, 4, None).to(dtype), want, dev, dtype)
    assert norm <= 1 and element <= 1
    for mistake in ["one part"] + (["scores", "values", "weights", "two parts", "half"] if dtype == torch.float32 else []):
        assert P.excess(in_fp32(q, k, v, 4, mistake).to(dtype), want, dev, dtype)[0] > 1, mistake


def test_one_rounding_is_predicted():
    x = torch.randn(20000, generator=torch.Generator().manual_seed(1)).double()
    err = torch.sqrt(((x.to(torch.bfloat16).double() - x) ** 2).sum() / (P.rounding(x, torch.bfloat16) ** 2).sum())
    assert abs(float(err) - 1) < 0.03
