"""Paged decode attention through a window, in batches of which a wave walks many units: the jump from the first tokens to the window
inside a share, masks of units that are refilled meanwhile, rows behind all that of NaN.  Against the definition in 64 bits."""
import numpy as np
import pytest
import torch

from tests import paged_bounds as P
from tests import paged_reference as R
from tests.test_gpu_paged import B, DT, ints, make_pool, randn, run_decode, tables  # noqa: F401  (B: the fixture)

pytestmark = pytest.mark.gpu
WAVES = 1024


def share(lens, window, sinks, items, unit):
    """Units that a wave walks: those of a request hold its first tokens or begin at the window's edge, and there is one at least."""
    total = 0
    for n in lens:
        edge = max(n - window, 0) if window else 0
        first = -(-min(sinks, edge) // unit)
        total += max(first + max(-(-n // unit) - max(edge // unit, first), 0), 1)
    return -(-total * items // WAVES)


def check(B, dt, hq, hk, d, lens, page, window, sinks, least, holes=0.0, n_pages=None, pool="rows", seed=0):
    unit = 32 if dt == "bf16" else 16
    group = hq // hk
    items = hk * -(-group // (16 if group <= 16 else 32))
    assert share(lens, window, sinks, items, unit) >= least, "the batch is too small for what this is about"
    rng = np.random.default_rng(seed)
    if n_pages is None:
        table, n_pages = tables(rng, lens, page)
    else:      # requests share pages
        table = rng.integers(0, n_pages, (len(lens), -(-max(lens) // page)))
    if holes:
        table[rng.random(table.shape) < holes] = -1
    keys = [[j for j in R.visible(n, window, sinks) if 0 <= table[r, j // page] < n_pages] for r, n in enumerate(lens)]
    seen = torch.zeros(n_pages, page, dtype=torch.bool)
    for r, at in enumerate(keys):
        at = np.asarray(at, dtype=np.int64)
        seen[table[r][at // page], at % page] = True
    kp, vp = make_pool(n_pages, page, hk, d, DT[dt], pool, seed)
    kp[~seen.cuda()] = float("nan")
    vp[~seen.cuda()] = float("nan")
    q = randn(len(lens), hq, d, seed=seed + 5, dtype=DT[dt])
    got = run_decode(B, B.make_shape(hq, hk, d, dt, 1e4), q.cuda(), kp, vp, ints(table), ints(lens), window, sinks)
    want, dev = P.decode_batch(q, kp.cpu(), vp.cpu(), table, keys, group)
    for r, n in enumerate(lens):
        if len(keys[r]) == 0:
            assert (got[r] == 0).all(), r
            continue
        norm, element = P.excess(got[r], want[r], dev[r], DT[dt])
        assert element <= 1 and (len(keys[r]) > 1000 or norm <= 1), (r, n, norm, element)


def lengths(seed, n, lo, hi, empty=3):
    lens = np.random.default_rng(seed).integers(lo, hi, n)
    lens[np.random.default_rng(seed + 1).permutation(n)[:empty]] = 0
    return lens.tolist()


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("page", [8, 16, 64, 256])
@pytest.mark.parametrize("window,sinks", [(2000, 70), (2000, 0), (311, 1000), (1, 1500)])
def test_windows_over_shares_of_many_units(B, dt, page, window, sinks):
    check(B, dt, 4, 2, 64, lengths(page, 40, 500, 9000), page, window, sinks, 2, seed=page + window)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("page", [8, 32])
def test_windows_over_shares_longer_than_a_register_of_page_ids(B, dt, page):
    """More than 16 units of pages of 8 (32 in fp32) to a wave: 64 page ids."""
    check(B, dt, 8, 8, 64, lengths(page, 60, 1500, 3500), page, 1400, 90, 17 if dt == "bf16" else 33, n_pages=1000, seed=page)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_windows_over_more_requests_than_lanes(B, dt):
    check(B, dt, 4, 2, 64, lengths(1, 200, 0, 900), 16, 400, 37, 2, seed=1)
    check(B, dt, 2, 1, 128, lengths(2, 131, 0, 1200), 32, 500, 3, 2, seed=2)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("hq", [20, 40])
def test_windows_under_more_heads_than_a_tile(B, dt, hq):
    check(B, dt, hq, 1, 128, lengths(hq, 90, 100, 1500), 16, 700, 40, 2, seed=hq)
    check(B, dt, 2 * hq, 2, 64, lengths(hq + 1, 30, 100, 3000), 8, 1200, 200, 2, seed=hq)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("page", [8, 64])
def test_windows_over_tables_with_holes(B, dt, page):
    check(B, dt, 4, 2, 64, lengths(page, 40, 500, 5000), page, 1900, 150, 2, holes=0.25, seed=page)
    check(B, dt, 4, 2, 64, lengths(page, 40, 500, 5000), page, 0, 0, 2, holes=0.25, seed=page)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("pool", ["heads", "together", "wide"])
def test_windows_over_pools_of_any_strides(B, dt, pool):
    check(B, dt, 4, 2, 128, lengths(4, 40, 500, 4000), 16, 1500, 45, 2, pool=pool, seed=4)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("page", [8, 16, 64])
def test_the_window_of_a_length_beyond_the_table(B, dt, page):
    """The window's edge is the length's, not the table's: of the rows that the table holds those in front of it are not seen, and where
    the whole window lies behind them there are only the first tokens, or nothing."""
    blocks, d = 320 // page, 64
    rows = blocks * page
    lens = [rows - 1, rows, rows + 1, rows + 70, rows + 149, rows + 150, rows + 151, 5 * rows, 2 ** 31 - 1]
    table = np.random.default_rng(page).permutation(len(lens) * blocks).reshape(len(lens), blocks)
    kp, vp = make_pool(len(lens) * blocks, page, 2, d, DT[dt], "rows", 3)
    q = randn(len(lens), 4, d, seed=5, dtype=DT[dt])
    for window, sinks in ((150, 0), (150, 20), (150, 3000), (1, 0), (1, 1), (2 ** 31 - 1, 0), (0, 5)):
        got = run_decode(B, B.make_shape(4, 2, d, dt, 1e4), q.cuda(), kp, vp, ints(table), ints(lens), window, sinks)
        keys = [[j for j in range(min(n, rows)) if window == 0 or j >= n - window or j < sinks] for n in lens]
        want, dev = P.decode_batch(q, kp.cpu(), vp.cpu(), table, keys, 2)
        for r in range(len(lens)):
            if keys[r]:
                assert P.excess(got[r], want[r], dev[r], DT[dt])[1] <= 1, (window, sinks, lens[r])
            else:
                assert (got[r] == 0).all(), (window, sinks, lens[r])
