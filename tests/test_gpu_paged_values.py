"""Paged decode attention where the values of its inputs are hard: weights that cancel, scores far from zero, infinite values and
values near the largest, each against the definition in 64 bits."""
import math

import numpy as np
import pytest
import torch

from tests import paged_bounds as P
from tests.test_gpu_paged import B, DT, ints, make_pool, randn, run_decode, tables  # noqa: F401  (B: the fixture)

pytestmark = pytest.mark.gpu
BOTH = pytest.mark.parametrize("dt", ["bf16", "f32"])


# ---- weights -------------------------------------------------------------------------------------------------------------------


@BOTH
@pytest.mark.parametrize("d", [64, 128])
def test_weights_keep_the_bits_of_fp32(B, dt, d):
    """Three keys of weights 1, w and about 1 - w with values 1, -1 and -1: what is left is what the weights lost.

    Scores of one product of powers of two and sums of two exact ones, all exact.  A weight is off by its argument (|x| <= 4.4 log2
    units, three roundings: 3 * 4.4 * ln 2 = 9.2 steps of 2^-24) and its exponential (2 steps); the weighted sum by at most 9 additions
    of two steps each, on something of size 1; the sum of weights is 2: (11.2 * 1 + 18) / 2 = 14.6 steps, and one rounding of the result."""
    n = 64
    w = torch.linspace(0.05, 0.95, n).double()
    q = torch.zeros(n, 2, d, dtype=DT[dt])
    q[..., 0] = q[..., 5] = 1.0
    kp = torch.zeros(n, 8, 1, d, dtype=DT[dt])
    for j, x in ((1, w), (2, 1 - w)):
        s = math.sqrt(d) * torch.log(x)
        kp[:, j, 0, 0] = s.to(torch.bfloat16).to(DT[dt])
        kp[:, j, 0, 5] = (s - kp[:, j, 0, 0].double()).to(torch.bfloat16).to(DT[dt])
    vp = torch.ones(n, 8, 1, d, dtype=DT[dt])
    vp[:, 1:] = -1.0
    got = run_decode(B, B.make_shape(2, 1, d, dt, 1e4), q.cuda(), kp.cuda(), vp.cuda(), ints(np.arange(n)[:, None]), ints([3] * n), 0, 0).cpu().double()
    s = (kp[:, :3, 0, 0].double() + kp[:, :3, 0, 5].double()) / math.sqrt(d)
    p = torch.softmax(s, 1)
    want = (p[:, 0] - p[:, 1] - p[:, 2])[:, None, None].expand_as(got)
    assert want.abs().max() < 2.0 ** -7
    err = (got - want).abs() - torch.finfo(DT[dt]).eps / 2 * want.abs() * 1.01
    assert float(err.max()) <= 14.6 * 2.0 ** -24, float(err.max()) * 2.0 ** 24


@BOTH
@pytest.mark.parametrize("d,hq,hk,page", [(64, 8, 2, 16), (128, 8, 2, 8), (128, 20, 1, 64), (64, 40, 1, 32), (128, 4, 4, 256)])
def test_errors_are_those_of_single_precision(B, dt, d, hq, hk, page):
    """The norm of the error and every element of it, for data whose roundings are independent (tests/test_paged_bounds.py shows
    that operands or weights of 16 bits would be noticed)."""
    lens = [7, 60, 513, 33, 300]
    table, n_pages = tables(np.random.default_rng(d + hq), lens, page)
    kp, vp = make_pool(n_pages, page, hk, d, DT[dt], "rows", hq)
    q = randn(len(lens), hq, d, seed=d, dtype=DT[dt], scale=0.5)
    got = run_decode(B, B.make_shape(hq, hk, d, dt, 1e4), q.cuda(), kp, vp, ints(table), ints(lens), 0, 0)
    want, dev = P.decode_batch(q, kp.cpu(), vp.cpu(), table, [range(n) for n in lens], hq // hk)
    for r, n in enumerate(lens):
        norm, element = P.excess(got[r], want[r], dev[r], DT[dt])
        assert norm <= 1 and element <= 1, (n, norm, element)


# ---- scores far from zero ----------------------------------------------------------------------------------------------------------


@BOTH
@pytest.mark.parametrize("d", [64, 128])
def test_the_only_key_has_weight_one_whatever_its_score(B, dt, d):
    """One visible row per request: its value is the result, bit for bit (a weight that is a power of two, divided by itself).  Scores of
    either sign up to d * 2^118, also one whose product with the scale is far from an fp32 number: 39936^2 * d."""
    sizes = [0.0, 2.0 ** -60, 1.0, 39936.0, 3.0 * 2 ** 20, 1.7e9, 2.0 ** 40, 1.1e15, 5.0e17]
    sizes = [x for x in sizes for _ in (0, 1)]
    n = len(sizes)
    size = torch.tensor(sizes)
    sign = torch.tensor([1.0, -1.0] * (n // 2))
    noise = 1 + torch.rand(n, 1, d, generator=torch.Generator().manual_seed(d)) / 8
    noise[6:8] = 1.0   # as it stands
    q = (size[:, None, None] * noise).to(DT[dt]).expand(n, 4, d).contiguous()
    for page in (8, 64):
        kp, vp = make_pool(n, page, 1, d, DT[dt], "rows", page)
        kp[:, 0, 0] = (size * sign).cuda().to(DT[dt])[:, None]
        got = run_decode(B, B.make_shape(4, 1, d, dt, 1e4), q.cuda(), kp, vp, ints(np.arange(n)[:, None]), ints([1] * n), 0, 0)
        assert torch.equal(got, vp[:, 0].expand(n, 4, d))


@BOTH
@pytest.mark.parametrize("lens", [[5], [40, 3, 700], [40000], [900] * 60], ids=str)
def test_equal_keys_share_the_weight_whatever_their_score(B, dt, lens):
    """Every third key equal and the others with half its score, which gives them no weight, or twice it where scores are negative: the
    mean of the values, over shares of several units and joined pieces.  Sums: as in tests/paged_reference.py."""
    d, page = 64, 16
    table, n_pages = tables(np.random.default_rng(1), lens, page)
    kp, vp = make_pool(n_pages, page, 1, d, DT[dt], "rows", 3)
    for size, sign in ((39936.0, 1.0), (39936.0, -1.0), (1.1e15, 1.0), (1.1e15, -1.0)):
        q = torch.full((len(lens), 2, d), size, dtype=DT[dt])
        low = 0.5 if sign > 0 else 2.0
        k = torch.full((n_pages * page, 1, d), size * sign * low, dtype=DT[dt])
        top = []
        for r, n in enumerate(lens):
            rows = torch.as_tensor(table[r][np.arange(0, n, 3) // page] * page + np.arange(0, n, 3) % page)
            k[rows] = size * sign
            top.append(rows)
        kp.copy_(k.view_as(kp))
        got = run_decode(B, B.make_shape(2, 1, d, dt, 1e4), q.cuda(), kp, vp, ints(table), ints(lens), 0, 0).cpu().double()
        v = vp.cpu().double().view(-1, d)
        for r, rows in enumerate(top):
            want, n = v[rows].mean(0), lens[r]
            bound = torch.finfo(DT[dt]).eps / 2 * want.abs() * 1.01 + 2 * (n / 16 + 64) * 2.0 ** -24 * v[rows].abs().mean(0)
            assert bool(((got[r] - want).abs() <= bound).all()), (size, sign, r)


# ---- values near the largest ---------------------------------------------------------------------------------------------------------


@BOTH
def test_values_near_the_largest_do_not_overflow(B, dt):
    """One key of each request has a weight 2^7 times that of the others and values of half the largest, and comes when others have
    been seen already or first of all: weights of at most 1 keep the sums in range.  64 requests of 1024 rows: shares of two units or more."""
    n, length, d, page = 64, 1024, 64, 64
    rng = np.random.default_rng(3)
    table, n_pages = tables(rng, [length] * n, page)
    kp = torch.zeros(n_pages, page, 1, d, dtype=DT[dt])
    vp = randn(n_pages, page, 1, d, seed=1, dtype=DT[dt])
    q = torch.zeros(n, 2, d, dtype=DT[dt])
    q[..., 0] = 1.0
    big = torch.full((d,), 1.7e38)
    big[1::2] *= -1
    at = [16 * r + 3 for r in range(n)]
    for r in range(n):
        kp[table[r, at[r] // page], at[r] % page, 0, 0] = 7 * math.log(2) * math.sqrt(d)
        vp[table[r, at[r] // page], at[r] % page, 0] = big.to(DT[dt])
    got = run_decode(B, B.make_shape(2, 1, d, dt, 1e4), q.cuda(), kp.cuda(), vp.cuda(), ints(table), ints([length] * n), 0, 0)
    want, dev = P.decode_batch(q, kp, vp, table, [range(length)] * n, 2)
    assert P.excess(got, want, dev, DT[dt])[1] <= 1


@BOTH
def test_a_single_largest_value_is_itself(B, dt):
    top = torch.finfo(DT[dt]).max
    kp, vp = make_pool(2, 8, 1, 64, DT[dt], "rows", 1)
    vp[:] = top
    q = randn(2, 3, 64, seed=2, dtype=DT[dt])
    got = run_decode(B, B.make_shape(3, 1, 64, dt, 1e4), q.cuda(), kp, vp, ints([[0], [1]]), ints([1, 1]), 0, 0)
    assert (got == top).all()


# ---- infinite values -----------------------------------------------------------------------------------------------------------------


@BOTH
@pytest.mark.parametrize("d,page,lens", [(64, 8, [1, 2, 5, 40]), (128, 16, [700, 33, 1]), (128, 64, [3000, 90]), (64, 32, [900] * 60)], ids=str)
def test_infinite_values_reach_the_result(B, dt, d, page, lens):
    """A visible value of +-inf makes its channel +-inf, both signs in one channel make NaN, and the other channels do not notice; weights of any
    bits, 1 among them.  What is not visible is infinite everywhere."""
    hq, hk, n = 6, 2, len(lens)
    table, n_pages = tables(np.random.default_rng(d), lens, page)
    kp, vp = make_pool(n_pages, page, hk, d, DT[dt], "rows", 3)
    q = randn(n, hq, d, seed=5, dtype=DT[dt])
    k, v = kp.cpu(), vp.cpu()
    seen = torch.zeros(n_pages, page, dtype=torch.bool)
    for r, length in enumerate(lens):
        seen[table[r][np.arange(length) // page], np.arange(length) % page] = True
    finite = v.clone()
    v[~seen] = float("inf")
    special = {}
    rng = np.random.default_rng(9)
    for r, length in enumerate(lens):
        for channel, values in ((3, [1]), (d - 2, [-1]), (17, [1, -1]), (40, [-1, -1])):
            rows = rng.permutation(length)[:len(values)]
            for j, x in zip(rows, values):
                v[table[r, j // page], j % page, :, channel] = x * float("inf")
            special[r, channel] = sum(x * float("inf") for x in values[:len(rows)])
    got = run_decode(B, B.make_shape(hq, hk, d, dt, 1e4), q.cuda(), kp, v.cuda(), ints(table), ints(lens), 0, 0).cpu().double()
    want, dev = P.decode_batch(q, k, finite, table, [range(x) for x in lens], hq // hk)
    for (r, channel), x in special.items():
        at = got[r, :, channel]
        assert bool(torch.isnan(at).all()) if math.isnan(x) else bool((at == x).all()), (r, channel, x, at)
        got[r, :, channel] = want[r, :, channel]
    assert P.excess(got, want, dev, DT[dt])[1] <= 1
