"""The calls over a paged cache in 8 bits with enough rows for the other side of each rule of their launches: streamed loads and stores, workgroups of
several tokens' queries, workgroups of both kinds mixed."""
import numpy as np
import pytest
import torch

from tests import paged_q8_reference as Q
from tests import paged_reference as R
from tests.test_gpu_paged import DT, ints, randn
from tests.test_gpu_paged_q8 import EPS, Pool

pytestmark = pytest.mark.gpu
PAGE = 32


@pytest.fixture(scope="module")
def B():
    from paper_2410_07590_amd import binding
    binding.lib()
    return binding


def runs_among(rng, n):
    """Slots of n tokens, -1 but for runs of 1 to 40 tokens, the first and the last token among them; 64 rows of the pool for each run."""
    count = 40
    slots, pool = np.full(n, -1, np.int64), rng.permutation(2 * count)
    for r in range(count):
        length, cached = int(rng.integers(1, 41)), int(rng.integers(0, 24))
        row = cached + np.arange(length)
        room = n // count
        at = 0 if r == 0 else n - length if r == count - 1 else r * room + int(rng.integers(0, room - length + 1))
        slots[at:at + length] = pool[2 * r + row // PAGE] * PAGE + row % PAGE
    return slots, 2 * count


@pytest.mark.parametrize("dt,hq,hk,d,n,layout,rot,norm,together,streamed", [
    # tokens' queries to a workgroup: as many as have 2048 units of 16 bytes between them, eight at most
    ("bf16", 32, 2, 128, 30801, 1, 96, True, 4, True), ("bf16", 16, 1, 128, 61501, 0, 128, True, 8, True),
    ("bf16", 81, 3, 64, 24301, 1, 64, False, 2, True), ("bf16", 64, 2, 64, 30727, 0, 32, True, 4, True),
    ("f32", 16, 2, 128, 30803, 1, 128, True, 4, True), ("f32", 40, 2, 128, 12301, 0, 48, False, 1, True),
    ("f32", 16, 1, 64, 61443, 1, 32, True, 8, True), ("f32", 64, 2, 64, 15401, 0, 64, True, 2, True),
    ("bf16", 6, 2, 64, 8193, 1, 64, True, 8, False), ("f32", 3, 1, 128, 8199, 0, 32, True, 8, False), ("bf16", 7, 7, 128, 16391, 1, 128, False, 8, False)])
def test_append_of_many_tokens(B, dt, hq, hk, d, n, layout, rot, norm, together, streamed):
    """Queries bit for bit those of the append in the shape's type, and some of them, keys and values against the definitions."""
    dtype, e = DT[dt], 2 if dt == "bf16" else 4
    assert (n * hq * d * e >= 240 << 20) == streamed
    tile = 1
    while tile < 8 and hq * d * e // 16 * tile * 2 <= 2048 and n >= 2048 * tile:
        tile *= 2
    assert tile == together
    rng = np.random.default_rng(n)
    slots, n_pages = runs_among(rng, n)
    q, k, v = (randn(n, h, d, seed=n + i, dtype=dtype) for i, h in enumerate((hq, hk, hk)))
    qw, kw = (randn(d, seed=n + 5 + i, dtype=dtype) if norm else None for i in (0, 1))
    pos = torch.from_numpy(rng.integers(0, 100000, n))
    gs, rotary, freq = B.make_shape(hq, hk, d, dt, 1e6, layout), B.tr_rotary_init(layout, rot, 1e6), R.frequencies(rot, 1e6)
    on_gpu = lambda t: None if t is None else t.cuda()   # noqa: E731
    gq, at = q.cuda(), ints(pos)
    out, same = (torch.full_like(gq, float("nan")) for _ in range(2))
    pool = Pool(B, n_pages, PAGE, hk, d, seed=3)
    B.tr_paged_append_q8(gs, rotary, gq, k.cuda(), v.cuda(), on_gpu(qw), on_gpu(kw), EPS, at, ints(slots), out, pool.pages)
    B.tr_paged_append(gs, rotary, gq, None, None, on_gpu(qw), None, EPS, at, None, same, None)
    torch.cuda.synchronize()
    assert torch.equal(out, same)
    some = np.unique(np.concatenate([np.arange(9), n - 1 - np.arange(9), rng.integers(0, n, 200)]))
    want, size = R.heads(q[some], qw, EPS, pos[some], freq, layout)
    R.assert_within(out.cpu()[some], want, R.heads_bound(want, size, dtype), "queries")
    held = np.flatnonzero(slots >= 0)
    keys, size = R.heads(k[held], kw, EPS, pos[held], freq, layout)
    pool.check(keys, 26 * 2.0 ** -24 * size + 1e-37, v[held], slots[held])


@pytest.mark.parametrize("dt,hk,d,page,order", [("bf16", 8, 128, 64, "rows"), ("bf16", 3, 64, 16, "heads"), ("bf16", 1, 128, 32, "rows"), ("f32", 4, 64, 32, "rows"),
                                                ("f32", 3, 128, 16, "heads"), ("f32", 4, 128, 64, "wide")])
def test_read_back_of_many_rows(B, dt, hk, d, page, order):
    """Results of 256 MiB and more: streamed.  Some pages are none; rows between the requests stay.  Compared on the GPU, in fp32, which is exact."""
    rng = np.random.default_rng(hk + d)
    row = hk * d * (2 if dt == "bf16" else 4)
    n_req, n_pages, rows = 37, 300, (128 << 20) // row + 1001
    cuts = np.sort(rng.choice(np.arange(1, rows), n_req - 1, replace=False))
    starts = np.concatenate([[3], cuts, [rows]])
    lens = np.maximum(np.diff(starts) - rng.integers(0, 50, n_req), 0)
    assert 2 * row * rows >= 256 << 20
    table = rng.integers(0, n_pages, (n_req, -(-int(lens.max()) // page)))
    table[rng.random(table.shape) < 0.01] = -1
    (k, ks), (v, vs) = (Q.random_pool(n_pages, page, hk, d, i, 3) for i in (1, 2))
    out = [torch.full((rows, hk, d), -3.0, dtype=DT[dt], device="cuda") for _ in range(2)]
    pages = B.make_pages_q8(Q.device_codes(k, order), Q.device_codes(v, order), ks.cuda(), vs.cuda())
    B.tr_paged_read_q8(B.make_shape(hk, hk, d, dt, 1e4), pages, ints(table), ints(lens), ints(starts), *out)
    torch.cuda.synchronize()
    for got, codes, scale in ((out[0], k, ks), (out[1], v, vs)):
        worth = Q.values(codes, scale).float().cuda()
        for r in range(n_req):
            j = torch.arange(int(lens[r]), device="cuda")
            p = torch.from_numpy(table[r]).cuda()[j // page]
            want = torch.where((p >= 0)[:, None, None], worth[p.clamp(min=0), j % page], 0.0)
            assert torch.equal(got[starts[r]:starts[r] + lens[r]].float(), want), r
            assert bool((got[starts[r] + lens[r]:starts[r + 1]] == -3).all()), r
        assert bool((got[:3] == -3).all())
