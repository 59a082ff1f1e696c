"""Writing a paged cache in 8 bits and reading it back, against the definitions in 64 bits."""
import numpy as np
import pytest
import torch

from tests import paged_q8_reference as Q
from tests import paged_reference as R

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f32": torch.float32}
EPS = 1e-6


@pytest.fixture(scope="module")
def B():
    from paper_2410_07590_amd import binding
    binding.lib()
    return binding


def ints(a):
    return torch.as_tensor(np.asarray(a), dtype=torch.int32).cuda()


def randn(*size, seed, dtype, scale=1.0):
    return (torch.randn(size, generator=torch.Generator().manual_seed(seed)) * scale).to(dtype)


class Pool:
    """A pool on the GPU and what it held before."""

    def __init__(self, B, n_pages, size, heads, d, order="rows", seed=0, spread=1):
        (self.k0, self.ks0), (self.v0, self.vs0) = (Q.random_pool(n_pages, size, heads, d, seed + i, spread) for i in (1, 2))
        self.k, self.v = Q.device_codes(self.k0, order), Q.device_codes(self.v0, order)
        self.ks, self.vs = self.ks0.cuda(), self.vs0.cuda()
        self.pages = B.make_pages_q8(self.k.view(torch.float8_e4m3fn), self.v.view(torch.float8_e4m3fn), self.ks, self.vs.view(torch.float8_e8m0fnu))

    def check(self, k, kerr, v, slots, what=""):
        torch.cuda.synchronize()
        Q.check_append(self.k.cpu(), self.ks.cpu(), self.k0, self.ks0, k, kerr, slots, what + " keys")
        Q.check_append(self.v.cpu(), self.vs.cpu(), self.v0, self.vs0, v.double(), 0, slots, what + " values")


def check_append(B, dt, hq, hk, d, slots, n_pages, page=16, rot=0, layout=1, norm=False, order="rows", packed=False, seed=0, scale=1.0, queries=True):
    dtype, n = DT[dt], len(slots)
    pool = Pool(B, n_pages, page, hk, d, order, seed)
    if packed:
        qkv = randn(n, hq + 2 * hk, d, seed=seed, dtype=dtype, scale=scale)
        q, k, v = qkv[:, :hq], qkv[:, hq:hq + hk], qkv[:, hq + hk:]
        gpu = qkv.cuda()
        gq, gk, gv = gpu[:, :hq], gpu[:, hq:hq + hk], gpu[:, hq + hk:]
    else:
        q, k, v = (randn(n, h, d, seed=seed + 3 * h + i, dtype=dtype, scale=scale) for i, h in enumerate((hq, hk, hk)))
        gq, gk, gv = q.cuda(), k.cuda(), v.cuda()
    pos = torch.randint(0, 100000, (n,), generator=torch.Generator().manual_seed(seed), dtype=torch.int32)
    qw, kw = (randn(d, seed=seed + i, dtype=dtype, scale=0.2) + 1 if norm else None for i in (50, 51))
    freq = R.frequencies(rot, 1e6)
    gs = B.make_shape(hq, hk, d, dt, 1e6, layout)
    out = torch.full((n, hq, d), float("nan"), dtype=dtype, device="cuda") if queries else None
    gpu_or_none = lambda t: None if t is None else t.cuda()   # noqa: E731
    B.tr_paged_append_q8(gs, B.tr_rotary_init(layout, rot, 1e6), gq if queries else None, gk, gv, gpu_or_none(qw) if queries else None, gpu_or_none(kw), EPS,
                         pos.cuda() if rot else None, ints(slots), out, pool.pages)
    keys, size = R.heads(k, kw, EPS, pos, freq, layout)
    exact = rot == 0 and not norm
    pool.check(k.double() if exact else keys, 0 if exact else 26 * 2.0 ** -24 * size + 1e-37, v, slots)
    if queries:
        want, size = R.heads(q, qw, EPS, pos, freq, layout)
        R.assert_within(out, want, R.heads_bound(want, size, dtype), "queries")


# ---- append ---------------------------------------------------------------------------------------------------------------------


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("layout", [0, 1])
@pytest.mark.parametrize("rot,norm", [(0, False), (0, True), (16, False), (48, True), (64, False), (64, True), (128, True)])
def test_append_types_layouts_and_parts_of_a_head(B, dt, d, layout, rot, norm):
    if rot > d:
        rot = 32
    slots, n_pages = Q.tokens_of(np.random.default_rng(rot + d), 5, 32, 70, 0, 40, 3)
    check_append(B, dt, 6, 2, d, slots, n_pages, 32, rot, layout, norm, seed=rot)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("hq,hk", [(1, 1), (28, 4), (32, 8), (5, 5), (6, 3), (40, 20), (64, 64)])
@pytest.mark.parametrize("new", [1, 2, 3, 5, 16, 33])
def test_append_head_counts_and_tokens_of_a_request(B, dt, hq, hk, new):
    slots, n_pages = Q.tokens_of(np.random.default_rng(hq + new), 7, 16, 50, new, new, 0)
    check_append(B, dt, hq, hk, 64 if hk > 8 else 128, slots, n_pages, 16, 64, seed=hk, packed=bool(new % 2))


@pytest.mark.parametrize("page", [16, 32, 64, 256, 1024])
@pytest.mark.parametrize("order", ["rows", "heads", "wide"])
def test_append_into_pools_of_any_layout(B, page, order):
    for dt, d in (("bf16", 128), ("f32", 64)):
        slots, n_pages = Q.tokens_of(np.random.default_rng(page), 4, page, 100, 1, 60, 2)
        check_append(B, dt, 4, 2, d, slots, n_pages, page, d, order=order, seed=page, norm=True)


@pytest.mark.parametrize("tokens", [1, 16, 17, 4000, 5001])
def test_append_one_prompt(B, tokens):
    for first in (0, 9):
        slots = np.arange(first, first + tokens)
        check_append(B, "bf16", 2, 1, 64, slots, -(-(tokens + first) // 32) + 1, 32, 64, seed=tokens, packed=True)


def test_append_many_requests_of_a_token(B):
    slots, n_pages = Q.tokens_of(np.random.default_rng(4), 3000, 16, 20, 1, 1, 100)
    check_append(B, "bf16", 2, 2, 64, slots, n_pages, 16, 64)
    slots, n_pages = Q.tokens_of(np.random.default_rng(4), 900, 16, 20, 0, 9, 100)
    check_append(B, "bf16", 2, 2, 64, slots, n_pages, 16, 64)


def test_append_without_queries_and_queries_alone(B):
    slots, n_pages = Q.tokens_of(np.random.default_rng(1), 4, 16, 30, 1, 40, 5)
    for dt in DT:
        check_append(B, dt, 4, 2, 128, slots, n_pages, 16, 128, queries=False)
    q = randn(9, 4, 128, seed=1, dtype=torch.bfloat16).cuda()
    gs = B.make_shape(4, 2, 128, "bf16", 1e6)
    out, want = torch.zeros_like(q), torch.zeros_like(q)
    B.tr_paged_append_q8(gs, None, q, None, None, None, None, EPS, ints(range(9)), None, out, None)
    B.tr_paged_append(gs, None, q, None, None, None, None, EPS, ints(range(9)), None, want, None)
    torch.cuda.synchronize()
    assert torch.equal(out, want)


def test_append_padding_other_pools_slots_and_rows_out_of_order(B):
    rng = np.random.default_rng(3)
    whole = np.arange(64)
    for slots in ([5 * 16 + 3], [-1, -1, 5 * 16 + 3, -1], [6 * 16, 6 * 16 + 1, 2 ** 31 - 1, 2 ** 31 - 17, 7], [-(2 ** 31), 0, -5, 17],
                  whole[::-1].copy(), np.concatenate([rng.permutation(16) + 16 * b for b in (3, 0, 2)]), [15, 14, 13, 20, 16, 40, 41, 33],
                  [16 * b + 7 for b in (5, 2, 0, 4, 1)]):
        check_append(B, "bf16", 3, 3, 64, np.asarray(slots), 6, 16, 64, seed=len(slots))
        check_append(B, "f32", 3, 3, 128, np.asarray(slots), 6, 16, 0, seed=len(slots))


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("size", [2.0 ** -140, 2.0 ** -20, 2.0 ** 9, 2.0 ** 60, 2.0 ** 118])
def test_append_of_values_of_any_size(B, dt, size):
    """Larger ones make what a block holds smaller codes, smaller ones become small codes themselves."""
    slots, n_pages = Q.tokens_of(np.random.default_rng(5), 9, 16, 40, 1, 20, 0)
    check_append(B, dt, 2, 2, 64, slots, n_pages, 16, 0, scale=size)
    if size > 2.0 ** -100:
        check_append(B, dt, 2, 2, 128, slots, n_pages, 16, 64, scale=size)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("first", [0, 5])
def test_append_of_zeros_the_largest_numbers_and_none(B, dt, first):
    """Blocks of zeros, of the largest finite numbers, with infinite and NaN channels, of the smallest numbers: each head by itself."""
    dtype, inf, nan = DT[dt], float("inf"), float("nan")
    k = randn(16 - first, 6, 64, seed=1, dtype=dtype)
    k[:, 0] = 0.0
    k[:, 1] = torch.finfo(dtype).max * torch.linspace(0.9, 1, 64)
    k[3, 2, 7], k[5, 2, 8], k[7, 2, 9] = inf, -inf, nan
    k[:, 3] = nan
    k[:, 4] = torch.finfo(dtype).tiny / 8
    k[2, 4, 3] = -torch.finfo(dtype).tiny
    k[2, 5, 3] = -torch.finfo(dtype).max
    v = k.flip(1).contiguous()
    pool = Pool(B, 2, 32, 6, 64, seed=5)
    slots = 32 + 16 + np.arange(first, 16)
    B.tr_paged_append_q8(B.make_shape(6, 6, 64, dt, 1e4), B.tr_rotary_init(1, 0, 1e4), None, k.cuda(), v.cuda(), None, None, EPS, None, ints(slots), None, pool.pages)
    pool.check(k.double(), 0, v, slots)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_a_block_filled_token_by_token_is_one_filled_at_once(B, dt):
    """The same scale; the same codes but for values that are below 2^-6 of a scale."""
    d, hk, n = 128, 4, 32
    k, v = (randn(n, hk, d, seed=s, dtype=DT[dt]) for s in (1, 2))
    grow = torch.linspace(-3, 6, n)[:, None, None]
    k, v = (k.float() * 2.0 ** grow).to(DT[dt]), (v.float() * 2.0 ** -grow).to(DT[dt])
    gs, rot = B.make_shape(hk, hk, d, dt, 1e4), B.tr_rotary_init(1, 0, 1e4)
    at_once, by_token, by_three = (Pool(B, 3, 16, hk, d, seed=9) for _ in range(3))
    B.tr_paged_append_q8(gs, rot, None, k.cuda(), v.cuda(), None, None, EPS, None, ints(range(16, 48)), None, at_once.pages)
    for pool, some in ((by_token, 1), (by_three, 3)):
        for t in range(0, n, some):
            m = min(some, n - t)
            B.tr_paged_append_q8(gs, rot, None, k[t:t + m].cuda(), v[t:t + m].cuda(), None, None, EPS, None, ints(range(16 + t, 16 + t + m)), None, pool.pages)
    torch.cuda.synchronize()
    at_once.check(k.double(), 0, v, np.arange(16, 48))
    for pool in (by_token, by_three):
        assert torch.equal(pool.ks, at_once.ks) and torch.equal(pool.vs, at_once.vs)
        for a, b in ((pool.k, at_once.k), (pool.v, at_once.v)):
            x, y = Q.VALUES[a.cpu().long()], Q.VALUES[b.cpu().long()]
            assert bool(((x == y) | (y.abs() < 2.0 ** -6)).all()) and bool(((x - y).abs() <= 2.0 ** -9).all())


def test_a_larger_row_changes_its_block_alone(B):
    """Held rows on both sides of the new one keep their values; every other byte of the pool is as it was."""
    for dt in DT:
        pool = Pool(B, 3, 32, 2, 64, seed=4)
        k, v = (randn(1, 2, 64, seed=s, dtype=DT[dt]) * 512 for s in (1, 2))
        v[:, 1] /= 2048   # this head's block has room for it
        slots = np.array([32 + 16 + 5])
        B.tr_paged_append_q8(B.make_shape(2, 2, 64, dt, 1e4), B.tr_rotary_init(1, 0, 1e4), None, k.cuda(), v.cuda(), None, None, EPS, None, ints(slots), None, pool.pages)
        pool.check(k.double(), 0, v, slots)
        assert (pool.ks.cpu() > pool.ks0).sum() == 2 and (pool.vs.cpu() > pool.vs0).sum() == 1


def test_append_of_no_tokens(B):
    pool = Pool(B, 2, 16, 2, 64)
    e = torch.empty(0, 2, 64, dtype=torch.bfloat16, device="cuda")
    B.tr_paged_append_q8(B.make_shape(2, 2, 64, "bf16", 1e4), None, e, e, e, None, None, EPS, ints([]), ints([]), e, pool.pages)
    pool.check(torch.zeros(0, 2, 64).double(), 0, torch.zeros(0, 2, 64), [])


# ---- read -----------------------------------------------------------------------------------------------------------------------


def run_read(B, dt, hk, d, k, v, ks, vs, table, lens, starts, n_rows, fill=-3.0):
    out = [torch.full((n_rows, hk, d), fill, dtype=DT[dt], device="cuda") for _ in range(2)]
    B.tr_paged_read_q8(B.make_shape(hk, hk, d, dt, 1e4), B.make_pages_q8(k, v, ks, vs), ints(table), ints(lens), ints(starts), *out)
    torch.cuda.synchronize()
    return [x.cpu().double() for x in out]


def check_read(B, dt, hk, d, lens, page, order="rows", starts=None, n_rows=None, holes=False, seed=0):
    rng = np.random.default_rng(seed)
    need = [-(-max(x, 0) // page) for x in lens]
    pool, at = rng.permutation(sum(need) + 2), 0
    table = np.full((len(lens), max(max(need, default=0), 1) + 1), 2 ** 31 - 1)
    for r, n in enumerate(need):
        table[r, :n] = pool[at:at + n]
        at += n
    if holes:
        table[rng.random(table.shape) < 0.3] = -1
    (k, ks), (v, vs) = (Q.random_pool(len(pool), page, hk, d, seed + i, 3) for i in (1, 2))
    if starts is None:
        starts = np.concatenate([[0], np.cumsum(np.maximum(lens, 0))])
    n_rows = int(starts[-1]) if n_rows is None else n_rows
    got = run_read(B, dt, hk, d, Q.device_codes(k, order), Q.device_codes(v, order), ks.cuda(), vs.cuda(), table, lens, starts, n_rows)
    for side, codes, scale in ((0, k, ks), (1, v, vs)):
        worth = Q.values(codes, scale)
        want = torch.full((n_rows, hk, d), -3.0, dtype=torch.float64)
        for r, length in enumerate(lens):
            for j in range(max(length, 0)):
                t = int(starts[r]) + j
                if t < starts[r + 1] and t < n_rows and j // page < table.shape[1]:
                    p = table[r, j // page]
                    want[t] = worth[p, j % page] if 0 <= p < len(pool) else 0.0
        assert torch.equal(got[side], want), (side, (got[side] != want).nonzero()[:3].tolist())


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("hk,d", [(1, 64), (3, 64), (4, 128), (8, 128), (40, 64)])
@pytest.mark.parametrize("page", [16, 64, 1024])
def test_read_back(B, dt, hk, d, page):
    check_read(B, dt, hk, d, [5, 0, 1, 16, 17, 33, 250], page, "rows", seed=page + hk)


@pytest.mark.parametrize("order", ["heads", "wide"])
def test_read_back_of_other_layouts_with_holes(B, order):
    check_read(B, "bf16", 3, 128, [100, 7, 0, 64, 65], 32, order, holes=True)
    check_read(B, "f32", 2, 64, [100, 7, 0, 64, 65], 16, order, holes=True, seed=1)


def test_read_back_into_part_of_a_cache(B):
    """Rows between, in front of and behind the requests' stay; lengths beyond their room, the table's and the outputs'; negative ones."""
    lens = [20, 40, -3, 7, 0, 60]
    check_read(B, "bf16", 2, 64, lens, 16, starts=np.array([3, 30, 55, 60, 70, 70, 200]), n_rows=100)
    check_read(B, "bf16", 2, 64, lens, 16, starts=np.array([3, 30, 55, 60, 70, 70, 200]), n_rows=71)
    check_read(B, "f32", 2, 64, lens, 32, starts=np.array([0, 0, 0, 0, 0, 0, 61]), n_rows=61)
    check_read(B, "f32", 2, 64, [50], 16, starts=np.array([2 ** 31 - 10, 2 ** 31 - 1]), n_rows=5)
    page, n = 16, 3
    k, ks = Q.random_pool(4, page, 1, 64, 1)
    got = run_read(B, "bf16", 1, 64, k.cuda(), k.cuda(), ks.cuda(), ks.cuda(), np.array([[2, 1]] * n), [2 ** 31 - 1] * n, [0, 40, 80, 120], 130)
    worth = Q.values(k, ks)[[2, 1]].flatten(0, 1)
    for r in range(n):
        assert torch.equal(got[0][40 * r:40 * r + 32], worth) and bool((got[0][40 * r + 32:40 * r + 40] == -3).all())


def test_read_back_of_many_requests(B):
    rng = np.random.default_rng(2)
    check_read(B, "bf16", 1, 64, rng.integers(0, 4, 5000).tolist(), 16, seed=3)
    check_read(B, "bf16", 1, 64, [0] * 700 + [3] + [0] * 500 + [40] + [0] * 90, 16, seed=3)


def test_read_back_of_every_code_at_every_scale(B):
    """256 codes x the scales that an append writes, of keys; values are the same codes at the opposite scales."""
    n = 256
    codes = torch.arange(256, dtype=torch.uint8).view(4, 64).repeat(4, 1)[None, :, None].expand(n, 16, 1, 64).contiguous()
    s = torch.arange(n).clamp(10, 247).to(torch.uint8)
    ks, vs = s.view(n, 1, 1).contiguous(), s.flip(0).view(n, 1, 1).contiguous()
    for dt in DT:
        got = run_read(B, dt, 1, 64, codes.cuda(), codes.cuda(), ks.cuda(), vs.cuda(), np.arange(n)[:, None], [16] * n, 16 * np.arange(n + 1), 16 * n)
        for side, scale in enumerate((ks, vs)):
            want = Q.values(codes, scale).reshape(16 * n, 1, 64)
            big = want.abs() >= 2.0 ** 128   # what an append never leaves: codes above 240 at the largest scale
            assert int(big[~big.isnan()].sum()) == int(big.sum())
            ok = (got[side] == want) | (torch.isnan(got[side]) & torch.isnan(want)) | (big & ~torch.isfinite(got[side]))
            assert bool(ok.all())


def test_read_back_of_nothing(B):
    pool = Pool(B, 2, 16, 2, 64)
    gs = B.make_shape(2, 2, 64, "bf16", 1e4)
    none, out = torch.empty(0, 2, 64, dtype=torch.bfloat16, device="cuda"), torch.ones(5, 2, 64, dtype=torch.bfloat16, device="cuda")
    B.tr_paged_read_q8(gs, pool.pages, ints(np.zeros((3, 1))), ints([1, 1, 1]), ints([0, 1, 2, 3]), none, none.clone())
    B.tr_paged_read_q8(gs, pool.pages, torch.empty(0, 4, dtype=torch.int32, device="cuda"), ints([]), ints([0]), out, out.clone())
    B.tr_paged_read_q8(gs, pool.pages, torch.empty(3, 0, dtype=torch.int32, device="cuda"), ints([1, 1, 1]), ints([0, 1, 2, 3]), out, out.clone())
    torch.cuda.synchronize()
    assert bool((out == 1).all())
