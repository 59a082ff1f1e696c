"""The calls over a paged cache in 8 bits at the ends of what they take: as many requests as there may be, heads whose squares are beyond fp32, positions
far away, queries that are not numbers."""
import numpy as np
import pytest
import torch

from tests import paged_q8_reference as Q
from tests import paged_reference as R
from tests.test_gpu_paged import DT, ints, randn, tables
from tests.test_gpu_paged_q8 import EPS, Pool, check_append, check_read
from tests.test_gpu_paged_q8_decode import check as check_decode
from tests.test_gpu_paged_q8_decode import run

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2410_07590_amd import binding
    binding.lib()
    return binding


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("size", [2.0 ** -70, 2.0 ** -30, 2.0 ** 60, 2.0 ** 68, 2.0 ** 100])
def test_append_norms_heads_whose_squares_are_beyond_fp32(B, dt, size):
    slots, n_pages = Q.tokens_of(np.random.default_rng(5), 6, 16, 40, 1, 20, 2)
    for d, layout, rot in ((64, 0, 64), (128, 1, 128), (128, 0, 32), (64, 1, 48)):
        check_append(B, dt, 4, 2, d, slots, n_pages, 16, rot, layout, norm=True, scale=size, seed=d)


def test_append_far_positions_and_scaled_frequencies(B):
    pos = np.array([0, 1, 2 ** 31 - 1, 2 ** 31 - 2, -1, -(2 ** 31), 10 ** 6, 123456789])
    slots = np.arange(3, 11)
    for layout in (0, 1):
        for dt, d, rot in (("f32", 64, 64), ("bf16", 128, 128), ("bf16", 128, 32)):
            freq = R.frequencies(rot, 1e6, "parts", 16.0, 8192)
            q, k, v = (randn(8, h, d, seed=h, dtype=DT[dt]) for h in (4, 2, 2))
            pool, out = Pool(B, 2, 16, 2, d, seed=3), torch.zeros_like(q).cuda()
            rotary = B.tr_rotary_init(layout, rot, 1e6, B.TR_SCALE_PARTS, 16.0, 8192, 1.0, 32.0, 1.277)
            B.tr_paged_append_q8(B.make_shape(4, 2, d, dt, 1e6, layout), rotary, q.cuda(), k.cuda(), v.cuda(), None, None, EPS, ints(pos), ints(slots), out, pool.pages)
            want, size = R.heads(k, None, EPS, torch.from_numpy(pos), freq, layout, 1.277)
            pool.check(want, 26 * 2.0 ** -24 * size + 1e-37, v, slots)
            want, size = R.heads(q, None, EPS, torch.from_numpy(pos), freq, layout, 1.277)
            R.assert_within(out, want, R.heads_bound(want, size, DT[dt]), "queries")


def test_a_head_of_nan_and_one_of_zeros_under_a_norm(B):
    for dt in DT:
        k, v = (randn(16, 3, 64, seed=s, dtype=DT[dt]) for s in (1, 2))
        k[4, 1, 9], k[5, 1] = float("nan"), 0.0
        w = randn(64, seed=4, dtype=DT[dt])
        pool, slots = Pool(B, 1, 16, 3, 64, seed=3), np.arange(16)
        B.tr_paged_append_q8(B.make_shape(3, 3, 64, dt, 1e4), B.tr_rotary_init(1, 32, 1e4), None, k.cuda(), v.cuda(), None, w.cuda(), EPS, ints(np.arange(16)), ints(slots),
                             None, pool.pages)
        want, size = R.heads(k, w, EPS, torch.arange(16), R.frequencies(32, 1e4), 1)
        assert torch.isnan(want[4, 1]).all()
        size[4, 1] = 0.0
        pool.check(want, 26 * 2.0 ** -24 * size + 1e-37, v, slots)


@pytest.mark.parametrize("n", [1, 2, 62, 63, 64, 65, 66, 126, 127, 128, 129, 4095, 4096, 4097])
def test_read_back_of_numbers_of_requests_around_a_waves_lanes(B, n):
    rng = np.random.default_rng(n)
    check_read(B, "bf16", 2, 64, rng.integers(0, 3, n).tolist(), 16, seed=n)
    check_read(B, "f32", 1, 64, [0] * (n - 1) + [70], 32, seed=n)
    check_read(B, "bf16", 3, 64, [35] + [0] * (n - 1), 16, seed=n, starts=np.array([2, 37] + [37] * (n - 1)), n_rows=50)


def test_read_back_of_as_many_requests_as_there_may_be(B):
    n = 65536
    g = torch.Generator().manual_seed(1)
    lens = torch.randint(0, 3, (n,), generator=g, dtype=torch.int32)
    starts = torch.cat([torch.zeros(1, dtype=torch.int32), lens.cumsum(0).to(torch.int32)])
    k, ks = Q.random_pool(512, 16, 1, 64, 3)
    table = torch.randint(0, 512, (n, 1), generator=g, dtype=torch.int32)
    out = [torch.zeros(int(starts[-1]), 1, 64, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    B.tr_paged_read_q8(B.make_shape(1, 1, 64, "bf16", 1e4), B.make_pages_q8(k.cuda(), k.cuda(), ks.cuda(), ks.cuda()), table.cuda(), lens.cuda(), starts.cuda(), *out)
    owner = torch.repeat_interleave(torch.arange(n), lens.long())
    row = torch.arange(len(owner)) - starts[owner].long()
    want = Q.values(k, ks)[table[owner, 0].long(), row]
    assert torch.equal(out[0].cpu().double(), want) and torch.equal(out[1], out[0])


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_decode_as_many_requests_as_there_may_be(B, dt):
    """65536 requests of no key or of one, whose value is the result."""
    n = 65536
    g = torch.Generator().manual_seed(1)
    lens = torch.randint(0, 2, (n,), generator=g, dtype=torch.int32)
    (k, ks), (v, vs) = (Q.random_pool(2048, 16, 1, 64, i) for i in (1, 2))
    table = torch.randint(0, 2048, (n, 5), generator=g, dtype=torch.int32)
    q = randn(n, 2, 64, seed=5, dtype=DT[dt])
    got = run(B, B.make_shape(2, 1, 64, dt, 1e4), q.cuda(), k.cuda(), v.cuda(), ks.cuda(), vs.cuda(), table.cuda(), lens.cuda())
    want = (Q.values(v, vs)[table[:, 0].long(), 0] * lens[:, None, None]).expand(n, 2, 64).cuda()
    if dt == "bf16":   # rounding to bf16 takes away what the weight is off
        assert torch.equal(got.double(), want)
    else:              # p v (1 + e1), e1 of up to two steps of the matrix unit, times 1 / p (1 + e2), (1 + e3): four steps of 2^-24
        assert ((got.double() - want).abs() <= 4.01 * 2.0 ** -24 * want.abs()).all()


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_decode_queries_that_are_not_numbers_stay_by_themselves(B, dt):
    hq, hk, d, lens = 6, 2, 128, [200, 3, 77]
    table, n_pages = tables(np.random.default_rng(1), lens, 16)
    (k, ks), (v, vs) = (Q.random_pool(n_pages, 16, hk, d, i) for i in (1, 2))
    q = randn(3, hq, d, seed=5, dtype=DT[dt])
    gs = B.make_shape(hq, hk, d, dt, 1e4)
    args = (k.cuda(), v.cuda(), ks.cuda(), vs.cuda(), ints(table), ints(lens))
    clean = run(B, gs, q.cuda(), *args)
    for bad in (float("nan"), float("inf"), -float("inf")):
        broken = q.clone()
        broken[0, 1, 5] = broken[1, 4, 127] = bad
        got = run(B, gs, broken.cuda(), *args)
        torch.cuda.synchronize()
        same = torch.ones(3, hq, dtype=torch.bool)
        same[0, 1] = same[1, 4] = False
        assert torch.equal(got[same.cuda()], clean[same.cuda()])
        if bad != bad:
            assert torch.isnan(got[~same.cuda()]).all()


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("wrong", ["apart", "twice", "often"])
def test_slots_that_are_not_side_by_side_leave_the_other_blocks_alone(B, dt, wrong):
    """Block 2 is named in two places, a row of it twice, or one row by 40 tokens: it holds anything, all others what they should."""
    good = [np.arange(3, 9), 16 * 5 + np.arange(16), 16 * 3 + np.array([7]), 16 * 1 + np.arange(4), 16 * 4 + np.arange(16)]
    bad = {"apart": [32 + np.arange(5), 32 + 9 + np.arange(4)], "twice": [32 + np.array([0, 1, 1, 2])], "often": [32 + np.full(40, 6)]}[wrong]
    slots = np.concatenate([good[0], bad[0], good[1], good[2], bad[-1] if wrong == "apart" else [], good[3], good[4]]).astype(np.int64)
    k, v = (randn(len(slots), 2, 64, seed=s, dtype=DT[dt]) for s in (1, 2))
    pool = Pool(B, 3, 32, 2, 64, seed=7)
    B.tr_paged_append_q8(B.make_shape(2, 2, 64, dt, 1e4), B.tr_rotary_init(1, 0, 1e4), None, k.cuda(), v.cuda(), None, None, EPS, None, ints(slots), None, pool.pages)
    torch.cuda.synchronize()
    for codes, scale, codes0, scale0 in ((pool.k, pool.ks, pool.k0, pool.ks0), (pool.v, pool.vs, pool.v0, pool.vs0)):   # block 2: as it was
        codes[1, :16].copy_(codes0[1, :16])
        scale[1, :, 0].copy_(scale0[1, :, 0])
    pool.check(k.double(), 0, v, np.where(slots // 16 == 2, -1, slots))


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("d,rot", [(64, 64), (64, 32), (128, 128), (128, 48), (128, 0)])
@pytest.mark.parametrize("layout", [0, 1])
def test_queries_are_those_of_the_append_in_the_shapes_type(B, dt, d, rot, layout):
    """Bit for bit: the same products in the same order."""
    n = 3000
    q = randn(n, 5, d, seed=rot, dtype=DT[dt]).cuda()
    w, pos = randn(d, seed=3, dtype=DT[dt]).cuda(), ints(np.arange(n) * 7)
    gs, rotary = B.make_shape(5, 5, d, dt, 1e4, layout), B.tr_rotary_init(layout, rot, 1e4)
    for norm in (None, w):
        a, b = torch.empty_like(q), torch.empty_like(q)
        B.tr_paged_append(gs, rotary, q, None, None, norm, None, EPS, pos, None, a, None)
        B.tr_paged_append_q8(gs, rotary, q, None, None, norm, None, EPS, pos, None, b, None)
        torch.cuda.synchronize()
        assert torch.equal(a, b)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("hq,hk", [(2, 2), (3, 3), (8, 4), (6, 6), (20, 10), (36, 2), (80, 2)])
@pytest.mark.parametrize("order", ["rows", "wide", "heads"])
def test_decode_heads_that_share_lines(B, dt, hq, hk, order):
    """64 channels: pairs of heads are shared out together where they lie in one line.  Few units and many, shares that cut items and that do not."""
    rng = np.random.default_rng(hq)
    for lens in ([1], [64], [65], [130, 0, 1], [700], list(rng.integers(0, 300, 9)), list(rng.integers(0, 200, 150)), [9000, 3], [64 * 40] * 13):
        check_decode(B, dt, hq, hk, 64, [int(x) for x in lens], page=32, order=order, seed=len(lens), hide=len(lens) < 20)
    check_decode(B, dt, hq, hk, 64, [5000, 70, 900], page=16, order=order, window=700, sinks=70, seed=5)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
def test_decode_bits_do_not_depend_on_the_tables_width(B, dt, d):
    lens = [5000, 1, 777, 2000]
    table, n_pages = tables(np.random.default_rng(1), lens, 16)
    (k, ks), (v, vs) = (Q.random_pool(n_pages, 16, 2, d, i) for i in (1, 2))
    q = randn(4, 8, d, seed=5, dtype=DT[dt]).cuda()
    gs, pool = B.make_shape(8, 2, d, dt, 1e4), (k.cuda(), v.cuda(), ks.cuda(), vs.cuda())
    want = run(B, gs, q, *pool, ints(table), ints(lens))
    for more in (1, 7, 300):   # columns that no length reaches
        assert torch.equal(want, run(B, gs, q, *pool, ints(np.concatenate([table, np.full((4, more), 7)], 1)), ints(lens)))
