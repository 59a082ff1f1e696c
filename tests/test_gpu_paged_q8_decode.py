"""Decode attention over a paged cache in 8 bits, against its definition in 64 bits over what the codes are worth."""
import numpy as np
import pytest
import torch

from tests import paged_bounds as P
from tests import paged_q8_reference as Q
from tests import paged_reference as R
from tests.test_gpu_paged import DT, EDGES, ints, randn, tables

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2410_07590_amd import binding
    binding.lib()
    return binding


def run(B, gs, q, k, v, ks, vs, table, lens, window=0, sinks=0, stream=None):
    out = torch.full_like(q, float("nan"))
    ws = B.workspace(B.tr_paged_decode_attn_q8_workspace_size(gs, q.shape[0], table.shape[1], k.shape[1])).fill_(0xff)
    B.tr_paged_decode_attn_q8(gs, q, B.make_pages_q8(k, v, ks, vs), table, lens, window, sinks, out, ws, stream)
    return out


def check(B, dt, hq, hk, d, lens, page=16, window=0, sinks=0, order="rows", seed=0, scale=2.0, hide=True, spread=2):
    dtype = DT[dt]
    table, n_pages = tables(np.random.default_rng(seed), lens, page)
    (k, ks), (v, vs) = (Q.random_pool(n_pages, page, hk, d, seed + i, spread) for i in (1, 2))
    worth_k, worth_v = Q.values(k, ks), Q.values(v, vs)
    if hide:   # whatever is not visible is NaN, and so are the scales of blocks without a visible row
        seen = torch.zeros(n_pages, page, dtype=torch.bool)
        for r, length in enumerate(lens):
            for j in R.visible(length, window, sinks):
                seen[table[r, j // page], j % page] = True
        k[~seen], v[~seen] = 127, 255
        blocks = seen.reshape(n_pages, page // 16, 16).any(2)
        for s in (ks, vs):
            s.transpose(1, 2)[~blocks] = 255
    q = randn(len(lens), hq, d, seed=seed + 5, dtype=dtype, scale=scale)
    gs = B.make_shape(hq, hk, d, dt, 1e4)
    got = run(B, gs, q.cuda(), Q.device_codes(k, order), Q.device_codes(v, order), ks.cuda(), vs.cuda(), ints(table), ints(lens), window, sinks)
    torch.cuda.synchronize()
    want, bound = R.decode_batch(q, worth_k, worth_v, torch.from_numpy(table), lens, window, sinks, hq // hk)
    R.assert_within(got, want, torch.finfo(dtype).eps / 2 * want.abs() * (1 + 2.0 ** -8) + bound + 1e-37, "attention")


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("page", [16, 32, 64, 256, 1024])
def test_lengths_at_every_edge(B, dt, d, page):
    check(B, dt, 8, 2, d, EDGES, page=page, seed=page + d)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("hq,hk", [(1, 1), (4, 4), (14, 2), (16, 1), (17, 1), (32, 1), (33, 1), (40, 1), (128, 1), (20, 10)])
def test_groups_of_heads(B, dt, hq, hk):
    check(B, dt, hq, hk, 128, [1, 0, 40, 300, 129], seed=hq)
    check(B, dt, hq, hk, 64, [700], page=64, seed=hq)


@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (5, 3), (16, 0), (31, 33), (32, 32), (33, 4), (100, 1), (128, 64), (257, 130), (5000, 7),
                                          (2 ** 31 - 1, 2 ** 31 - 1), (40, 2 ** 31 - 1), (0, 9)])
@pytest.mark.parametrize("page", [16, 32, 128])
def test_windows_and_first_tokens(B, window, sinks, page):
    check(B, "bf16", 6, 2, 128, EDGES, page=page, window=window, sinks=sinks, seed=page)
    check(B, "f32", 2, 2, 64, EDGES, page=page, window=window, sinks=sinks, seed=page)


@pytest.mark.parametrize("order", ["heads", "wide"])
@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_pools_of_any_strides(B, order, dt):
    check(B, dt, 8, 2, 64, [300, 17, 0, 129], order=order, page=32, window=100, sinks=5, seed=2)
    check(B, dt, 4, 1, 128, [300, 17, 0, 129], order=order, page=16, seed=3)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_long_and_many(B, dt):
    check(B, dt, 4, 2, 64, [20011], seed=1, hide=False)
    check(B, dt, 4, 2, 128, [9000, 3, 5001, 0, 77], seed=2, hide=False, page=64)
    check(B, dt, 2, 1, 64, list(np.random.default_rng(0).integers(0, 70, 700)), seed=3, hide=False)
    check(B, dt, 2, 2, 64, [9, 4000] + [1] * 300, seed=4, hide=False)
    check(B, dt, 16, 4, 64, list(np.random.default_rng(5).integers(0, 400, 300)), seed=5, hide=False)
    check(B, dt, 34, 1, 64, list(np.random.default_rng(6).integers(0, 300, 70)), seed=6, hide=False)
    check(B, dt, 1, 1, 64, [0, 700] * 20 + list(np.random.default_rng(7).integers(0, 30, 5000)) + [900], seed=7, hide=False)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("page", [16, 32])
def test_shares_longer_than_a_register_of_page_ids(B, dt, page):
    """Requests that share pages: 64 rows of 9000 keys over a pool of 500 pages, so every wave walks many units; some pages are none."""
    rng = np.random.default_rng(page)
    n, d, n_pages = 64, 64, 500
    lens = rng.integers(8800, 9200, n)
    table = rng.integers(0, n_pages, (n, -(-9200 // page)))
    table[rng.random(table.shape) < 0.02] = -1
    (k, ks), (v, vs) = (Q.random_pool(n_pages, page, 1, d, 3 + i, 2) for i in (1, 2))
    q = randn(n, 2, d, seed=5, dtype=DT[dt], scale=2.0)
    for window, sinks in ((0, 0), (3000, 100)):
        got = run(B, B.make_shape(2, 1, d, dt, 1e4), q.cuda(), k.cuda(), v.cuda(), ks.cuda(), vs.cuda(), ints(table), ints(lens), window, sinks)
        want, bound = R.decode_batch(q, Q.values(k, ks), Q.values(v, vs), torch.from_numpy(table), lens, window, sinks, 2)
        R.assert_within(got, want, torch.finfo(DT[dt]).eps / 2 * want.abs() * 1.01 + bound, "shared pages")


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("hq,hk,page", [(8, 2, 16), (34, 1, 32)])
def test_errors_are_those_of_single_precision(B, dt, d, hq, hk, page):
    """Operands and weights of fewer bits would show in the norm of the error."""
    lens = [700, 1, 4000, 65]
    table, n_pages = tables(np.random.default_rng(1), lens, page)
    (k, ks), (v, vs) = (Q.random_pool(n_pages, page, hk, d, i, 1) for i in (1, 2))
    q = randn(len(lens), hq, d, seed=5, dtype=DT[dt])
    got = run(B, B.make_shape(hq, hk, d, dt, 1e4), q.cuda(), k.cuda(), v.cuda(), ks.cuda(), vs.cuda(), ints(table), ints(lens))
    torch.cuda.synchronize()
    want, dev = P.decode_batch(q, Q.values(k, ks), Q.values(v, vs), table, [range(x) for x in lens], hq // hk)
    norm, most = P.excess(got, want, dev, DT[dt])
    assert norm <= 1 and most <= 1, (norm, most)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_a_key_that_outweighs_all_others_and_scales_of_any_size(B, dt):
    """Scores far from zero; values of blocks whose scales are 2^60 apart."""
    for lens in ([700], [64, 1, 33]):
        check(B, dt, 4, 2, 128, lens, seed=3, scale=300.0, spread=6)
        check(B, dt, 4, 2, 64, lens, seed=4, scale=0.0, spread=30)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("at", [0, 15, 16, 31, 40])
def test_a_nan_stays_with_its_head_or_channel(B, dt, at):
    hq, hk, d, lens = 8, 2, 64, [41, 41]
    table, n_pages = tables(np.random.default_rng(1), lens, 16)
    (k, ks), (v, vs) = (Q.random_pool(n_pages, 16, hk, d, i, 1) for i in (1, 2))
    q = randn(2, hq, d, seed=5, dtype=DT[dt])
    gs = B.make_shape(hq, hk, d, dt, 1e4)
    args = (ints(table), ints(lens))
    clean = run(B, gs, q.cuda(), k.cuda(), v.cuda(), ks.cuda(), vs.cuda(), *args)
    k[table[0, at // 16], at % 16, 1, 9] = 127
    v[table[0, at // 16], at % 16, 0, 5] = 255
    got = run(B, gs, q.cuda(), k.cuda(), v.cuda(), ks.cuda(), vs.cuda(), *args)
    torch.cuda.synchronize()
    assert torch.isnan(got[0, 4:]).all() and torch.isnan(got[0, :4, 5]).all()
    got[0, 4:], got[0, :4, 5] = clean[0, 4:], clean[0, :4, 5]
    assert torch.equal(got, clean)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_pages_that_are_none_and_lengths_outside_the_table(B, dt):
    hq, hk, d, page = 4, 2, 64, 16
    table = np.array([[0, -1, 2, 5], [2 ** 31 - 1, 7, -5, 1], [-1, -1, -1, -1], [3, 4, 1, 0], [1, 2, 3, 4]])
    lens = [60, 50, 64, 2 ** 31 - 1, -4]
    (k, ks), (v, vs) = (Q.random_pool(7, page, hk, d, i, 1) for i in (1, 2))
    q = randn(5, hq, d, seed=5, dtype=DT[dt])
    for window, sinks in ((0, 0), (2 ** 31 - 1 - 50, 3), (20, 5)):
        got = run(B, B.make_shape(hq, hk, d, dt, 1e4), q.cuda(), k.cuda(), v.cuda(), ks.cuda(), vs.cuda(), ints(table), ints(lens), window, sinks)
        torch.cuda.synchronize()
        wants = []
        for r, length in enumerate(lens):
            keys = [j for j in range(min(max(length, 0), 64)) if (window == 0 or j >= length - window or j < sinks) and 0 <= table[r, j // page] < 7]
            at = torch.tensor(keys, dtype=torch.long)
            p = torch.from_numpy(table[r])[at // page]
            wants.append(R.decode(q[r], Q.values(k, ks)[p, at % page], Q.values(v, vs)[p, at % page], keys, hq // hk))
        want, bound = (torch.stack([w[i] for w in wants]) for i in (0, 1))
        R.assert_within(got, want, torch.finfo(DT[dt]).eps / 2 * want.abs() * 1.01 + bound, "holes")


def test_into_its_own_queries_and_bit_for_bit_on_another_stream(B):
    hq, hk, d, lens = 8, 2, 128, [3000, 17, 0, 900]
    table, n_pages = tables(np.random.default_rng(1), lens, 32)
    pool = [x.cuda() for i in (1, 2) for x in Q.random_pool(n_pages, 32, hk, d, i, 1)]
    k, ks, v, vs = pool
    for dt in DT:
        q = randn(4, hq, d, seed=5, dtype=DT[dt]).cuda()
        gs = B.make_shape(hq, hk, d, dt, 1e4)
        want = run(B, gs, q, k, v, ks, vs, ints(table), ints(lens))
        side = torch.cuda.Stream()
        t, n = ints(table), ints(lens)
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            again = run(B, gs, q, k, v, ks, vs, t, n)
        own = q.clone()
        ws = B.workspace(B.tr_paged_decode_attn_q8_workspace_size(gs, 4, t.shape[1], 32))
        B.tr_paged_decode_attn_q8(gs, own, B.make_pages_q8(k, v, ks, vs), t, n, 0, 0, own, ws)
        torch.cuda.synchronize()
        assert torch.equal(again, want) and torch.equal(own, want)
