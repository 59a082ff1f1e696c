"""The paged cache's operators against their definitions in 64 bits: each by itself where it can go wrong, then together."""
import numpy as np
import pytest
import torch

from tests import helpers as H
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


# ---- block tables and slots --------------------------------------------------------------------------------------------------


def run_map(B, cached, new, first, page, free, table, n_slots, offset=0):
    n = len(cached)

    def room(m):  # filled with rubbish, and `offset` entries into an allocation
        return torch.full((m + offset,), -77, dtype=torch.int32, device="cuda")[offset:]
    tab = ints(table) if n else torch.empty((0, table.shape[1]), dtype=torch.int32, device="cuda")
    outs = dict(kv_lens=room(n), cu_new=room(n + 1), slots=room(n_slots), pos=room(n_slots), counts=room(2))
    B.tr_page_map(ints(cached), ints(new), None if first is None else ints(first), page, ints(free), tab, **outs)
    torch.cuda.synchronize()
    return [x.cpu().numpy().astype(np.int64) for x in (tab, outs["kv_lens"], outs["cu_new"], outs["slots"], outs["pos"], outs["counts"])]


def check_map(B, *args, offset=0):
    for name, got, want in zip(("table", "kv_lens", "cu_new", "slots", "pos", "counts"), run_map(B, *args, offset=offset), R.page_map(*args)):
        assert got.shape == want.shape and np.array_equal(got, want), (name, np.argwhere(got != want)[:5].tolist())


def batch(rng, n, page, cached_hi, new_hi, spare=3):
    cached, new = rng.integers(0, cached_hi + 1, n), rng.integers(0, new_hi + 1, n)
    have, need = -(-cached // page), -(-(cached + new) // page)
    pool = rng.permutation(int(need.sum()) + 5)
    table = np.full((n, int(need.max(initial=0)) + spare), -1)
    at = 0
    for r in range(n):
        table[r, :have[r]] = pool[at:at + have[r]]
        at += have[r]
    return cached, new, table, pool[at:]


@pytest.mark.parametrize("page", [8, 16, 128, 1024])
@pytest.mark.parametrize("n,cached_hi,new_hi,pad", [
    (1, 40, 1, 0), (1, 0, 5000, 9), (2, 3000, 1, 3), (63, 700, 40, 0), (64, 700, 1, 1), (65, 90, 300, 2), (257, 500, 30, 0), (1000, 60, 9, 5),
    (4096, 100, 3, 1)])
def test_map_of_a_batch(B, page, n, cached_hi, new_hi, pad):
    rng = np.random.default_rng(n + page)
    cached, new, table, free = batch(rng, n, page, cached_hi, new_hi)
    first = rng.integers(0, 9000, n) if n % 2 else None
    check_map(B, cached, new, first, page, free, table, int(new.sum()) + pad, offset=n % 4)


def test_map_without_requests_tokens_or_slots(B):
    check_map(B, [], [], None, 16, [4, 5], np.zeros((0, 3)), 6)
    check_map(B, [], [], None, 16, [], np.zeros((0, 0)), 0)
    check_map(B, [5, 0, 16], [0, 0, 0], None, 16, [], np.full((3, 2), 9), 4)
    check_map(B, [5, 0, 16], [20, 1, 1], None, 16, [7, 8, 9, 10], np.full((3, 2), 3), 0)     # pages are taken all the same
    check_map(B, [5, 0, 16], [20, 1, 9], [7, -4, 2 ** 31 - 3], 16, [7, 8, 9, 10], np.full((3, 2), 3), 25)  # fewer slots than tokens


def test_map_where_pages_or_columns_run_out_and_lengths_are_absurd(B):
    rng = np.random.default_rng(5)
    cached, new, table, free = batch(rng, 40, 16, 100, 60)
    total = int(new.sum())
    for n_free in (0, 1, 17, 60):
        check_map(B, cached, new, None, 16, free[:n_free], table, total)
    check_map(B, cached, new, None, 16, free, table[:, :4].copy(), total)
    check_map(B, cached, new, None, 16, free, np.where(rng.random(table.shape) < 0.3, -1, table), total)  # held pages that are none
    check_map(B, cached, new, None, 16, free, np.where(table >= 0, 2 ** 30, table), total)                # a slot beyond 31 bits
    cached, new = cached.copy(), new.copy()
    cached[3], new[4], cached[7], new[7] = -5, -(2 ** 31), -1, 3
    check_map(B, cached, new, None, 16, free, table, 3000)
    cached[11], new[11] = 2 ** 31 - 5, 40
    cached[12], new[12] = 2 ** 31 - 1, 2 ** 31 - 1
    check_map(B, cached, new, None, 16, free, table, 3000)


@pytest.mark.parametrize("page", [8, 16])
def test_map_of_more_pages_than_can_be_counted(B, page):
    # the sum of pages is cut within the ninth (17th) request: what is behind it gets no page, and no entry keeps its old one
    huge = 2 ** 31 - 1
    cached = np.array([3] + [0, 5, huge] * 12 + [4, page, 0])
    new = np.array([9] + [huge, huge, 7] * 12 + [30, 2 * page, 1])
    free, table = np.arange(50, 110), np.full((len(cached), 9), 3)
    check_map(B, cached, new, None, page, free, table, 2000)
    check_map(B, cached[::-1].copy(), new[::-1].copy(), None, page, free, table, 2000)
    check_map(B, np.zeros(4096, int), np.full(4096, huge), None, page, free, np.full((4096, 3), 3), 10)


# ---- heads into pages ------------------------------------------------------------------------------------------------------------


def make_pool(n_pages, page, hk, d, dtype, layout, seed, device="cuda"):
    """k, v [pages, page, heads, channels], views of differently laid out allocations."""
    if layout == "rows":
        k, v = (randn(n_pages, page, hk, d, seed=seed + i, dtype=dtype).to(device) for i in (0, 1))
    elif layout == "heads":       # the rows of a head lie together
        k, v = (randn(n_pages, hk, page, d, seed=seed + i, dtype=dtype).to(device).transpose(1, 2) for i in (0, 1))
    elif layout == "together":    # K and V of a page in one allocation
        kv = randn(n_pages, 2, page, hk, d, seed=seed, dtype=dtype).to(device)
        k, v = kv[:, 0], kv[:, 1]
    else:                         # heads and rows further apart than they need to be
        wide = randn(2, n_pages, page, hk + 1, d + 16, seed=seed, dtype=dtype).to(device)
        k, v = wide[0, :, :, :hk, :d], wide[1, :, :, :hk, :d]
    return k, v


def check_append(B, dt, hq, hk, d, tokens, rot, layout, norm=True, with_q=True, with_kv=True, packed=False, pool="rows", page=16, seed=0,
                 pos=None, slots=None, amplitude=1.0, freq=None, in_place=False, data=None, shape_rotary=False):
    dtype = DT[dt]
    n_pages = -(-tokens // page) + 2
    rng = np.random.default_rng(seed)
    if data is not None:
        q, k, v = data
    elif packed:
        qkv = randn(tokens, hq + 2 * hk, d, seed=seed, dtype=dtype)
        q, k, v = qkv[:, :hq], qkv[:, hq:hq + hk], qkv[:, hq + hk:]
    else:
        q, k, v = (randn(tokens, h, d, seed=seed + i, dtype=dtype) for i, h in enumerate((hq, hk, hk)))
    pos = rng.integers(0, 200000, tokens) if pos is None else np.asarray(pos)
    slots = rng.permutation(n_pages * page)[:tokens] if slots is None else np.asarray(slots)
    gs = B.make_shape(hq, hk, d, dt, 1e6, layout)
    if freq is None:
        freq = R.frequencies(rot, 1e6)
        rotary = None if shape_rotary else B.tr_rotary_init(layout, rot, 1e6, amplitude=amplitude)
    else:
        rotary = B.tr_rotary(layout, rot, amplitude)
        for m, f in enumerate(freq):
            rotary.freq[m] = f
    qw, kw = (randn(d, seed=seed + 7 + i, dtype=dtype) + 1 if norm else None for i in (0, 1))
    kp, vp = make_pool(n_pages, page, hk, d, dtype, pool, seed + 20)
    k0, v0 = kp.cpu().clone(), vp.cpu().clone()
    if packed and data is None:
        dev = qkv.cuda()
        dq, dk, dv = dev[:, :hq], dev[:, hq:hq + hk], dev[:, hq + hk:]
    else:
        dq, dk, dv = q.cuda(), k.cuda(), v.cuda()
    out = dq if in_place else torch.full((tokens, hq, d), float("nan"), dtype=dtype, device="cuda")
    cuda = lambda t: None if t is None else t.cuda()
    B.tr_paged_append(gs, rotary, dq if with_q else None, dk if with_kv else None, dv if with_kv else None, cuda(qw) if with_q else None, cuda(kw),
                      EPS, ints(pos) if rot else None, ints(slots) if with_kv else None, out if with_q else None,
                      B.make_pages(kp, vp) if with_kv else None)
    torch.cuda.synchronize()
    p = torch.from_numpy(pos.astype(np.int64))
    if with_q:
        want, size = R.heads(q, qw, EPS, p, freq, layout, amplitude)
        R.assert_within(out, want, R.heads_bound(want, size, dtype), "queries")
    k1, v1 = kp.cpu(), vp.cpu()
    if with_kv:
        want, size = R.heads(k, kw, EPS, p, freq, layout, amplitude)
        bound = R.heads_bound(want, size, dtype)
        for t, s in enumerate(slots):
            if 0 <= s < n_pages * page:
                R.assert_within(k1[s // page, s % page], want[t], bound[t], "key of token %d" % t)
                assert np.array_equal(H.bits_t(v1[s // page, s % page]), H.bits_t(v[t])), t
                k1[s // page, s % page], v1[s // page, s % page] = k0[s // page, s % page], v0[s // page, s % page]
    assert np.array_equal(H.bits_t(k1), H.bits_t(k0)) and np.array_equal(H.bits_t(v1), H.bits_t(v0)), "rows without a token changed"


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("layout", [0, 1])
@pytest.mark.parametrize("rot", [0, 16, 48, 64, 112, 128])
def test_append_types_layouts_and_parts_of_a_head(B, dt, d, layout, rot):
    if rot > d:
        pytest.skip("more channels than a head has")
    check_append(B, dt, 6, 2, d, 37, rot, layout, seed=rot + d)
    check_append(B, dt, 3, 1, d, 5, rot, layout, norm=False, seed=rot + d, amplitude=1.2772588722239782 if rot else 1.0)


@pytest.mark.parametrize("hq,hk", [(1, 1), (4, 4), (28, 4), (32, 8), (40, 40), (128, 1)])
@pytest.mark.parametrize("tokens", [1, 2, 130])
def test_append_head_counts_and_numbers_of_tokens(B, hq, hk, tokens):
    check_append(B, "bf16", hq, hk, 128, tokens, 128, 1, packed=True, seed=hq + tokens)
    check_append(B, "f32", hq, hk, 64, tokens, 32, 0, seed=hq + tokens, page=8)


@pytest.mark.parametrize("pool", ["rows", "heads", "together", "wide"])
@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_append_into_pools_of_any_strides(B, pool, dt):
    check_append(B, dt, 8, 2, 64, 50, 64, 1, pool=pool, page=32, seed=3)
    check_append(B, dt, 8, 1, 128, 50, 32, 0, pool=pool, page=8, packed=True, seed=4)


def test_append_with_the_norm_of_one_side(B):
    for which in (0, 1):
        gs = B.make_shape(4, 2, 128, "bf16", 1e4, 1)
        q, k, v = (randn(11, h, 128, seed=h, dtype=torch.bfloat16) for h in (4, 2, 2))
        w, p = randn(128, seed=9, dtype=torch.bfloat16), torch.arange(11) * 7
        kp, vp = make_pool(2, 16, 2, 128, torch.bfloat16, "rows", 3)
        out = torch.empty_like(q).cuda()
        B.tr_paged_append(gs, None, q.cuda(), k.cuda(), v.cuda(), w.cuda() if which == 0 else None, w.cuda() if which == 1 else None, EPS, ints(p),
                          ints(np.arange(11)), out, B.make_pages(kp, vp))
        for got, x, weight in ((out, q, w if which == 0 else None), (kp.flatten(0, 1)[:11], k, w if which == 1 else None)):
            want, size = R.heads(x, weight, EPS, p, R.frequencies(128, 1e4), 1)
            R.assert_within(got, want, R.heads_bound(want, size, torch.bfloat16), "norm of side %d" % which)


def test_append_many_tokens(B):
    check_append(B, "bf16", 5, 1, 64, 3001, 64, 1, packed=True, seed=9, page=64)


def test_append_one_side_only_and_in_place(B):
    check_append(B, "bf16", 6, 2, 128, 33, 128, 0, with_q=False, seed=1)
    check_append(B, "bf16", 6, 2, 128, 33, 128, 1, with_kv=False, seed=2)
    check_append(B, "bf16", 6, 2, 128, 33, 64, 1, in_place=True, seed=3)
    check_append(B, "f32", 6, 2, 64, 33, 64, 0, in_place=True, seed=4)
    check_append(B, "bf16", 6, 2, 128, 33, 128, 1, shape_rotary=True, seed=5)     # the shape's own layout and base
    check_append(B, "f32", 6, 2, 64, 33, 64, 0, shape_rotary=True, seed=6)


def test_append_padding_and_slots_outside_the_pool(B):
    page, tokens = 16, 40
    n_slots = (-(-tokens // page) + 2) * page
    slots = np.random.default_rng(1).permutation(n_slots)[:tokens]
    slots[[0, 7, 39]] = -1
    slots[[3, 20]] = [n_slots, 2 ** 31 - 1]
    slots[8] = -(2 ** 31)
    for dt, d in (("bf16", 128), ("f32", 64)):
        check_append(B, dt, 4, 2, d, tokens, 64, 1, slots=slots, page=page)
        check_append(B, dt, 4, 2, d, tokens, 64, 1, slots=np.full(tokens, -1), page=page)


def test_append_far_positions_and_scaled_frequencies(B):
    pos = np.array([0, 1, 2 ** 31 - 1, 2 ** 31 - 2, -1, -(2 ** 31), 10 ** 6, 123456789])
    for layout in (0, 1):
        check_append(B, "f32", 2, 1, 64, 8, 64, layout, pos=pos, seed=layout)
        check_append(B, "f32", 2, 1, 128, 8, 128, layout, pos=pos, freq=R.frequencies(128, 1e6, "parts", 16.0, 8192), amplitude=1.277, seed=5)
        check_append(B, "bf16", 2, 1, 128, 8, 32, layout, pos=pos, freq=np.linspace(0, 1, 16), seed=6)


def test_append_heads_of_any_size(B):
    """Zeros, values whose squares are far from one, a head of NaN among others."""
    for dt, d in (("bf16", 128), ("f32", 64)):
        q, k, v = (randn(9, h, d, seed=h, dtype=torch.float32) for h in (4, 2, 2))
        for x in (q, k):
            x[0] = 0.0
            x[1] *= 1e15
            x[2] *= 1e-12
            x[3, 1] *= 3e4
            x[4, 0, 5] = 1e17
        check_append(B, dt, 4, 2, d, 9, 32, 1, data=[x.to(DT[dt]) for x in (q, k, v)], seed=8)
    gs = B.make_shape(4, 2, 128, "bf16", 1e4)
    q = randn(3, 4, 128, seed=1, dtype=torch.bfloat16)
    clean, out = torch.empty_like(q).cuda(), torch.empty_like(q).cuda()
    w = torch.ones(128, dtype=torch.bfloat16).cuda()
    B.tr_paged_append(gs, None, q.cuda(), None, None, w, None, EPS, ints([1, 2, 3]), None, clean, None)
    q[1, 2, 77] = float("nan")
    B.tr_paged_append(gs, None, q.cuda(), None, None, w, None, EPS, ints([1, 2, 3]), None, out, None)
    torch.cuda.synchronize()
    assert torch.isnan(out[1, 2]).all()
    out[1, 2] = clean[1, 2]
    assert torch.equal(out, clean)


def test_append_without_norm_agrees_with_the_contiguous_append(B):
    """Same rows as tr_kv_append (64-bit products, one rounding), up to the rounding of fp32 products."""
    for dt, d, layout in (("bf16", 128, 0), ("bf16", 64, 1), ("f32", 128, 1)):
        gs = B.make_shape(8, 2, d, dt, 1e6, layout)
        k, v = (randn(48, 2, d, seed=s, dtype=DT[dt]).cuda() for s in (1, 2))
        pos = ints(np.arange(48) * 911)
        ck, cv, kp, vp = (torch.zeros(64, 2, d, dtype=DT[dt], device="cuda") for _ in range(4))
        B.tr_kv_append(gs, k, v, pos, ck, cv, 0)
        B.tr_paged_append(gs, None, None, k, v, None, None, EPS, pos, ints(np.arange(48)), None,
                          B.make_pages(kp.view(4, 16, 2, d), vp.view(4, 16, 2, d)))
        torch.cuda.synchronize()
        assert torch.equal(cv, vp)
        step = torch.finfo(DT[dt]).eps
        assert (ck.double() - kp.double()).abs().max() <= step * float(ck.double().abs().max())
        if dt == "bf16":
            assert (ck != kp).float().mean() < 1e-3


# ---- attention of one token -----------------------------------------------------------------------------------------------------


def tables(rng, lens, page, spare_cols=2, spare_pages=3):
    need = [-(-max(x, 0) // page) for x in lens]
    pool = rng.permutation(sum(need) + spare_pages)
    table = np.full((len(lens), max(need, default=0) + spare_cols), -1)
    at = 0
    for r, n in enumerate(need):
        table[r, :n] = pool[at:at + n]
        at += n
    return table, len(pool)


def run_decode(B, gs, q, kp, vp, table, lens, window, sinks, stream=None):
    out = torch.full_like(q, float("nan"))
    need = B.tr_paged_decode_attn_workspace_size(gs, q.shape[0], table.shape[1], kp.shape[1])
    ws = B.workspace(need).fill_(0xff)   # NaN in every type that partial results may have
    B.tr_paged_decode_attn(gs, q, B.make_pages(kp, vp), table, lens, window, sinks, out, ws, stream)
    return out


def check_decode(B, dt, hq, hk, d, lens, page=16, window=0, sinks=0, pool="rows", seed=0, scale=2.0, hide=True):
    dtype = DT[dt]
    rng = np.random.default_rng(seed)
    table, n_pages = tables(rng, lens, page)
    kp, vp = make_pool(n_pages, page, hk, d, dtype, pool, seed)
    if hide:   # whatever is not visible is NaN
        seen = torch.zeros(n_pages, page, dtype=torch.bool)
        for r, length in enumerate(lens):
            for j in R.visible(length, window, sinks):
                seen[table[r, j // page], j % page] = True
        kp[~seen.cuda()] = float("nan")
        vp[~seen.cuda()] = float("nan")
    q = randn(len(lens), hq, d, seed=seed + 5, dtype=dtype, scale=scale)
    gs = B.make_shape(hq, hk, d, dt, 1e4)
    got = run_decode(B, gs, q.cuda(), kp, vp, ints(table), ints(lens), window, sinks)
    torch.cuda.synchronize()
    want, bound = R.decode_batch(q, kp.cpu(), vp.cpu(), torch.from_numpy(table), lens, window, sinks, hq // hk)
    R.assert_within(got, want, torch.finfo(dtype).eps / 2 * want.abs() * (1 + 2.0 ** -8) + bound + 1e-37, "attention")


EDGES = [1, 2, 7, 8, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 0, 255, 256, 257, 0, 511, 513, 1000]


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("page", [8, 16, 32, 64, 256, 1024])
def test_decode_lengths_at_every_edge(B, dt, d, page):
    check_decode(B, dt, 8, 2, d, EDGES, page=page, seed=page + d)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("hq,hk", [(1, 1), (4, 4), (14, 2), (16, 1), (17, 1), (32, 1), (33, 1), (40, 1), (128, 1), (20, 10)])
def test_decode_groups_of_heads(B, dt, hq, hk):
    check_decode(B, dt, hq, hk, 128, [1, 0, 40, 300, 129], seed=hq)
    check_decode(B, dt, hq, hk, 64, [700], page=64, seed=hq)


@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (5, 3), (16, 0), (31, 33), (32, 32), (33, 4), (100, 1), (128, 64), (257, 130), (5000, 7),
                                          (2 ** 31 - 1, 2 ** 31 - 1), (40, 2 ** 31 - 1), (0, 9)])
@pytest.mark.parametrize("page", [8, 32, 128])
def test_decode_windows_and_first_tokens(B, window, sinks, page):
    check_decode(B, "bf16", 6, 2, 128, EDGES, page=page, window=window, sinks=sinks, seed=page)
    check_decode(B, "f32", 2, 2, 64, EDGES, page=page, window=window, sinks=sinks, seed=page)


@pytest.mark.parametrize("pool", ["heads", "together", "wide"])
@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_decode_over_pools_of_any_strides(B, pool, dt):
    check_decode(B, dt, 8, 2, 64, [300, 17, 0, 129], pool=pool, page=32, window=100, sinks=5, seed=2)
    check_decode(B, dt, 4, 1, 128, [300, 17, 0, 129], pool=pool, page=8, seed=3)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_decode_long_and_many(B, dt):
    check_decode(B, dt, 4, 2, 64, [20011], seed=1, hide=False)
    check_decode(B, dt, 4, 2, 128, [9000, 3, 5001, 0, 77], seed=2, hide=False, page=64)
    check_decode(B, dt, 2, 1, 64, list(np.random.default_rng(0).integers(0, 70, 700)), seed=3, hide=False)
    check_decode(B, dt, 2, 2, 64, [9, 4000] + [1] * 300, seed=4, hide=False)
    # pieces joined by the waves that begin them; more requests than a wave has lanes, by more than one each
    check_decode(B, dt, 16, 4, 64, list(np.random.default_rng(5).integers(0, 400, 300)), seed=5, hide=False)
    check_decode(B, dt, 34, 1, 64, list(np.random.default_rng(6).integers(0, 300, 70)), seed=6, hide=False)
    check_decode(B, dt, 1, 1, 64, [0, 700] * 20 + list(np.random.default_rng(7).integers(0, 30, 5000)) + [900], seed=7, hide=False)


def test_decode_many_requests_of_many_heads(B):
    """Rows of two blocks of query heads, joined by the waves that begin them."""
    check_decode(B, "bf16", 40, 1, 64, list(np.random.default_rng(8).integers(20, 90, 830)), seed=8, hide=False)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_decode_as_many_requests_as_there_may_be(B, dt):
    """65536 requests of no key or of one, whose value is the result."""
    n, page = 65536, 8
    lens = torch.randint(0, 2, (n,), generator=torch.Generator().manual_seed(1), dtype=torch.int32)
    kp, vp = make_pool(4096, page, 1, 64, DT[dt], "rows", 3)
    table = torch.randint(0, 4096, (n, 5), generator=torch.Generator().manual_seed(2), dtype=torch.int32)
    q = randn(n, 2, 64, seed=5, dtype=DT[dt])
    got = run_decode(B, B.make_shape(2, 1, 64, dt, 1e4), q.cuda(), kp, vp, table.cuda(), lens.cuda(), 0, 0)
    want = (vp[table[:, 0].long().cuda(), 0] * lens.cuda()[:, None, None]).expand(n, 2, 64)
    if dt == "bf16":   # the weight p is off by 2^-16 at most, which rounding to bf16 takes away
        assert torch.equal(got, want)
    else:              # p v (1 + e1), e1 of up to two steps of the matrix unit, times 1 / p (1 + e2), (1 + e3): four steps of 2^-24
        assert ((got.double() - want.double()).abs() <= 4.01 * 2.0 ** -24 * want.double().abs()).all()


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("page", [8, 16])
def test_decode_shares_longer_than_a_register_of_page_ids(B, dt, page):
    """Requests that share pages: 64 rows of 9000 keys over a pool of 500 pages, so every wave walks many units."""
    rng = np.random.default_rng(page)
    n, d, n_pages = 64, 64, 500
    lens = rng.integers(8800, 9200, n)
    table = rng.integers(0, n_pages, (n, -(-9200 // page)))
    table[rng.random(table.shape) < 0.02] = -1
    kp, vp = make_pool(n_pages, page, 1, d, DT[dt], "rows", 3)
    q = randn(n, 2, d, seed=5, dtype=DT[dt], scale=2.0)
    got = run_decode(B, B.make_shape(2, 1, d, dt, 1e4), q.cuda(), kp, vp, ints(table), ints(lens), 0, 0)
    want, bound = R.decode_batch(q, kp.cpu(), vp.cpu(), torch.from_numpy(table), lens, 0, 0, 2)
    R.assert_within(got, want, torch.finfo(DT[dt]).eps / 2 * want.abs() * 1.01 + bound, "shared pages")


def test_decode_scores_of_any_size(B):
    """One key that outweighs all others, at either end of a long row; scores far from zero on either side."""
    for dt, d in (("bf16", 128), ("f32", 64)):
        for lens in ([700], [64, 1, 33]):
            check_decode(B, dt, 4, 2, d, lens, seed=6, scale=30.0)
            check_decode(B, dt, 4, 2, d, lens, seed=7, scale=0.0)
        gs = B.make_shape(2, 1, d, dt, 1e4)
        for sign in (1.0, -1.0):
            kp, vp = make_pool(32, 16, 1, d, DT[dt], "rows", 1)
            kp[:] = (0.05 * kp.float()).to(DT[dt])
            kp[..., 0] += sign * 40.0      # every score near +-1700 log2 units
            table = torch.arange(32, dtype=torch.int32).view(1, 32)
            q = randn(1, 2, d, seed=3, dtype=DT[dt])
            q[..., 0] = 120.0 if d == 128 else 90.0
            for peak in (None, 0, 511, 260):
                k = kp.clone()
                if peak is not None:
                    k.view(512, d)[peak, 1] += 20.0
                got = run_decode(B, gs, q.cuda(), k, vp, table.cuda(), ints([512]), 0, 0)
                want, bound = R.decode_batch(q, k.cpu(), vp.cpu(), table, [512], 0, 0, 2)
                R.assert_within(got, want, torch.finfo(DT[dt]).eps / 2 * want.abs() * 1.01 + bound, "sign %g peak %s" % (sign, peak))


def test_decode_queries_that_are_not_numbers_stay_by_themselves(B):
    for dt, d in (("bf16", 128), ("f32", 64)):
        table, n_pages = tables(np.random.default_rng(2), [300, 90], 16)
        kp, vp = make_pool(n_pages, 16, 2, d, DT[dt], "rows", 3)
        q = randn(2, 8, d, seed=5, dtype=DT[dt])
        gs = B.make_shape(8, 2, d, dt, 1e4)
        clean = run_decode(B, gs, q.cuda(), kp, vp, ints(table), ints([300, 90]), 0, 0)
        q[0, 3, 7], q[1, 4] = float("nan"), float("inf")
        got = run_decode(B, gs, q.cuda(), kp, vp, ints(table), ints([300, 90]), 0, 0)
        assert torch.isnan(got[0, 3]).all() and torch.isnan(got[1, 4]).all()
        got[0, 3], got[1, 4] = clean[0, 3], clean[1, 4]
        assert torch.equal(got, clean)
        kp[int(table[1, 1]), 3, 1, 5] = float("nan")      # a visible key of one request and head
        got = run_decode(B, gs, q.cuda(), kp, vp, ints(table), ints([300, 90]), 0, 0)
        assert torch.isnan(got[1, 4:]).all() and not torch.isnan(got[1, :4]).any()
        got[0, 3], got[1, 4:] = clean[0, 3], clean[1, 4:]
        assert torch.equal(got, clean)


def test_decode_into_its_own_queries(B):
    for dt, d in (("bf16", 128), ("f32", 64)):
        lens = [5000, 3, 0, 200]
        table, n_pages = tables(np.random.default_rng(2), lens, 16)
        kp, vp = make_pool(n_pages, 16, 2, d, DT[dt], "rows", 3)
        q = randn(4, 8, d, seed=5, dtype=DT[dt]).cuda()
        gs = B.make_shape(8, 2, d, dt, 1e4)
        want = run_decode(B, gs, q, kp, vp, ints(table), ints(lens), 0, 0)
        B.tr_paged_decode_attn(gs, q, B.make_pages(kp, vp), ints(table), ints(lens), 0, 0, q,
                               B.workspace(B.tr_paged_decode_attn_workspace_size(gs, 4, table.shape[1], 16)))
        assert torch.equal(q, want)


def test_decode_pages_that_are_none(B):
    """Holes in the table: keys without a page have no weight; a request of holes only gets zeros."""
    rng = np.random.default_rng(4)
    for dt, hq, hk, d, page in (("bf16", 6, 2, 128, 8), ("bf16", 4, 1, 64, 16), ("f32", 4, 4, 64, 16), ("bf16", 4, 2, 128, 128)):
        lens = [500, 90, 33, 700, 8]
        table, n_pages = tables(rng, lens, page)
        table[rng.random(table.shape) < 0.3] = -1
        table[rng.random(table.shape) < 0.1] = n_pages
        table[rng.random(table.shape) < 0.1] = 2 ** 31 - 1
        table[rng.random(table.shape) < 0.1] = -(2 ** 31)
        table[2] = -1
        kp, vp = make_pool(n_pages, page, hk, d, DT[dt], "rows", 3)
        q = randn(len(lens), hq, d, seed=5, dtype=DT[dt])
        gs = B.make_shape(hq, hk, d, dt, 1e4)
        for window, sinks in ((0, 0), (130, 20)):
            got = run_decode(B, gs, q.cuda(), kp, vp, ints(table), ints(lens), window, sinks)
            want, bound = R.decode_batch(q, kp.cpu(), vp.cpu(), torch.from_numpy(table), lens, window, sinks, hq // hk)
            R.assert_within(got, want, torch.finfo(DT[dt]).eps / 2 * want.abs() * 1.01 + bound, "holes")
            assert (got[2] == 0).all()


def test_decode_lengths_outside_the_table(B):
    """Negative lengths are none; of a length beyond the table what the table holds is looked at."""
    lens = [-3, 200, 2 ** 31 - 1, -(2 ** 31)]
    table = np.random.default_rng(0).permutation(20).reshape(4, 5)
    kp, vp = make_pool(20, 16, 2, 64, torch.bfloat16, "rows", 3)
    q = randn(4, 4, 64, seed=5, dtype=torch.bfloat16)
    got = run_decode(B, B.make_shape(4, 2, 64, "bf16", 1e4), q.cuda(), kp, vp, ints(table), ints(lens), 0, 0)
    want, bound = R.decode_batch(q, kp.cpu(), vp.cpu(), torch.from_numpy(table), lens, 0, 0, 2)
    R.assert_within(got, want, 2.0 ** -8 * want.abs() * 1.01 + bound, "clipped lengths")
    empty = torch.empty((4, 0), dtype=torch.int32, device="cuda")
    got = run_decode(B, B.make_shape(4, 2, 64, "bf16", 1e4), q.cuda(), kp, vp, empty, ints(lens), 0, 0)
    assert (got == 0).all()


def test_offsets_beyond_32_bits(B):
    """A pool of more than 4 GiB each for K and V, the pages in use at its end."""
    page, hk, d = 64, 8, 128
    n_pages = (5 << 30) // (page * hk * d * 2)
    kp, vp = (torch.empty(n_pages, page, hk, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    lens, used = [190, 64], [n_pages - 1, 3, n_pages - 2, n_pages - 3]
    table = np.array([[used[0], used[1], used[2]], [used[3], -1, -1]])
    small_k, small_v = make_pool(4, page, hk, d, torch.bfloat16, "rows", 1, device="cpu")
    tokens = [(r, j) for r in (0, 1) for j in range(lens[r])]
    rows = [(used.index(table[r, j // page]), j % page) for r, j in tokens]
    k, v = (torch.stack([s[a] for a in rows]) for s in (small_k, small_v))
    gs = B.make_shape(16, hk, d, "bf16", 1e4)
    pages = B.make_pages(kp, vp)
    B.tr_paged_append(gs, B.tr_rotary_init(0, 0, 1e4), None, k.cuda(), v.cuda(), None, None, EPS, None,
                      ints([table[r, j // page] * page + j % page for r, j in tokens]), None, pages)
    for i, p in enumerate(used):
        n = 62 if i == 2 else 64
        assert torch.equal(kp[p, :n].cpu(), small_k[i, :n]) and torch.equal(vp[p, :n].cpu(), small_v[i, :n])
    q = randn(2, 16, d, seed=2, dtype=torch.bfloat16)
    got = run_decode(B, gs, q.cuda(), kp, vp, ints(table), ints(lens), 0, 0)
    where = torch.tensor([[0, 1, 2], [3, -1, -1]])
    want, bound = R.decode_batch(q, small_k, small_v, where, lens, 0, 0, 2)
    R.assert_within(got, want, 2.0 ** -8 * want.abs() * 1.01 + bound, "far pages")


def test_decode_repeats_bit_for_bit_and_on_another_stream(B):
    rng = np.random.default_rng(1)
    lens = [5000, 1, 777, 2000]
    table, n_pages = tables(rng, lens, 16)
    kp, vp = make_pool(n_pages, 16, 2, 128, torch.bfloat16, "rows", 3)
    q = randn(4, 8, 128, seed=5, dtype=torch.bfloat16).cuda()
    gs = B.make_shape(8, 2, 128, "bf16", 1e4)
    first = run_decode(B, gs, q, kp, vp, ints(table), ints(lens), 0, 0)
    wide = np.concatenate([table, np.full((4, 300), 7)], 1)   # columns that no length reaches
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        again = run_decode(B, gs, q, kp, vp, ints(table), ints(lens), 0, 0)
        wider = run_decode(B, gs, q, kp, vp, ints(wide), ints(lens), 0, 0)
    s.synchronize()
    handed = run_decode(B, gs, q, kp, vp, ints(table), ints(lens), 0, 0, stream=torch.cuda.current_stream())
    torch.cuda.synchronize()
    assert torch.equal(first, again) and torch.equal(first, wider) and torch.equal(first, handed)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_decodes_that_overlap_on_two_streams(B, dt):
    rng = np.random.default_rng(2)
    jobs = []
    for lens, page, hq, hk in (([4000, 30, 900], 16, 8, 2), ([20] * 200 + [3000], 64, 20, 1)):   # the second with two blocks of heads
        table, n_pages = tables(rng, lens, page)
        kp, vp = make_pool(n_pages, page, hk, 128, DT[dt], "rows", page)
        q, gs = randn(len(lens), hq, 128, seed=5, dtype=DT[dt]).cuda(), B.make_shape(hq, hk, 128, dt, 1e4)
        need = B.tr_paged_decode_attn_workspace_size(gs, len(lens), table.shape[1], page)
        alone = run_decode(B, gs, q, kp, vp, ints(table), ints(lens), 700, 3)
        jobs.append((gs, q, B.make_pages(kp, vp), ints(table), ints(lens), B.workspace(need), alone, [torch.empty_like(q) for _ in range(8)], torch.cuda.Stream()))
    torch.cuda.synchronize()
    for i in range(8):
        for gs, q, pool, table, lens, ws, _, outs, s in jobs:
            B.tr_paged_decode_attn(gs, q, pool, table, lens, 700, 3, outs[i], ws, s)
    torch.cuda.synchronize()
    for job in jobs:
        assert all(torch.equal(job[6], out) for out in job[7])


# ---- together --------------------------------------------------------------------------------------------------------------------


class Server:
    """Three requests whose caches grow in pages: prompts, then one token at a time; everything that a step reads and writes
    lies in buffers that a captured graph can keep."""

    def __init__(self, B, dt="bf16", page=16, room=40, seed=0):
        self.B, self.dtype, self.page, self.room = B, DT[dt], page, room
        self.hq, self.hk, self.d, self.rot, self.n = 6, 2, 128 if dt == "bf16" else 64, 32, 3
        self.gs = B.make_shape(self.hq, self.hk, self.d, dt, 1e4, 1)
        self.rotary = B.tr_rotary_init(1, self.rot, 1e4, B.TR_SCALE_PARTS, 4.0, 64, 1.0, 8.0, 1.13)
        self.freq = R.frequencies(self.rot, 1e4, "parts", 4.0, 64, 1.0, 8.0)
        rng = np.random.default_rng(seed)
        self.order = rng.permutation(64)
        self.kp, self.vp = make_pool(64, page, self.hk, self.d, self.dtype, "heads", seed)
        self.kp.fill_(float("nan"))
        self.vp.fill_(float("nan"))
        self.pages = B.make_pages(self.kp, self.vp)
        i32 = lambda *s: torch.zeros(*s, dtype=torch.int32, device="cuda")
        self.cached, self.new, self.lens, self.free = i32(3), i32(3), i32(3), i32(64)
        self.table = torch.full((3, 20), -1, dtype=torch.int32, device="cuda")
        self.cu, self.counts, self.slots, self.pos = i32(4), i32(2), i32(room), i32(room)
        blank = lambda h: torch.zeros(room, h, self.d, dtype=self.dtype, device="cuda")
        self.q, self.k, self.v, self.q_out = blank(self.hq), blank(self.hk), blank(self.hk), blank(self.hq)
        self.last, self.out = i32(3), torch.zeros(3, self.hq, self.d, dtype=self.dtype, device="cuda")
        self.qw, self.kw = (randn(self.d, seed=50 + i, dtype=self.dtype).cuda() for i in (0, 1))
        self.ws = B.workspace(B.tr_paged_decode_attn_workspace_size(self.gs, 3, 20, page))
        self.used, self.held = 0, [0, 0, 0]
        self.ks, self.vs = [[], [], []], [[], [], []]

    def load(self, new, seed):
        """The next step's tokens, in the host's program between steps."""
        total = sum(new)
        self.x = [randn(total, h, self.d, seed=seed + i, dtype=self.dtype) for i, h in enumerate((self.hq, self.hk, self.hk))]
        self.cached.copy_(ints(self.held))
        self.new.copy_(ints(new))
        self.free.copy_(ints(np.concatenate([self.order[self.used:], np.zeros(self.used)])))
        for dst, src in zip((self.q, self.k, self.v), self.x):
            dst[:total].copy_(src)
        self.last.copy_(ints(np.maximum(np.cumsum(new) - 1, 0)))
        self.step_new = new

    def step(self):
        B = self.B
        B.tr_page_map(self.cached, self.new, None, self.page, self.free, self.table, self.lens, self.cu, self.slots, self.pos, self.counts)
        B.tr_paged_append(self.gs, self.rotary, self.q, self.k, self.v, self.qw, self.kw, EPS, self.pos, self.slots, self.q_out, self.pages)
        B.tr_paged_decode_attn(self.gs, self.q_out[self.last.long()], self.pages, self.table, self.lens, 50, 3, self.out, self.ws)

    def check(self):
        torch.cuda.synchronize()
        q, k, v = self.x
        at = 0
        tokens, pages = self.counts.tolist()
        assert tokens == sum(self.step_new)
        for r, n in enumerate(self.step_new):
            pos = torch.arange(self.held[r], self.held[r] + n)
            want, size = R.heads(k[at:at + n], self.kw.cpu(), EPS, pos, self.freq, 1, 1.13)
            self.ks[r] += list(zip(want, R.heads_bound(want, size, self.dtype)))
            self.vs[r] += list(v[at:at + n])
            self.held[r] += n
            at += n
        self.used += pages
        table = self.table.cpu()
        assert self.lens.tolist() == self.held
        for r in range(3):
            if not self.held[r]:
                assert (self.out[r] == 0).all()
                continue
            rows = [(int(table[r, j // self.page]), j % self.page) for j in range(self.held[r])]
            kc, vc = (torch.stack([t[a].cpu() for a in rows]) for t in (self.kp, self.vp))
            for j in range(self.held[r]):
                R.assert_within(kc[j], *self.ks[r][j], "key %d of request %d" % (j, r))
                assert torch.equal(vc[j], self.vs[r][j])
            keys = R.visible(self.held[r], 50, 3)
            qr = self.q_out[int(self.last[r])].cpu()
            want, bound = R.decode(qr, kc[keys], vc[keys], keys, self.hq // self.hk)
            R.assert_within(self.out[r], want, torch.finfo(self.dtype).eps / 2 * want.abs() * 1.01 + bound, "request %d" % r)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_a_server_steps(B, dt):
    s = Server(B, dt)
    for i, new in enumerate([[17, 0, 3], [1, 0, 1], [1, 30, 1], [16, 1, 0], [1, 1, 1], [12, 12, 12], [1, 1, 1]]):
        s.load(new, 100 * i)
        s.step()
        s.check()


def test_a_captured_step_serves_other_lengths(B):
    s = Server(B)
    s.load([5, 2, 0], 1)
    s.step()
    s.check()
    s.load([1, 1, 1], 2)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        s.step()
    for i, new in enumerate([[1, 1, 1], [20, 0, 9], [0, 33, 1], [1, 1, 1], [14, 13, 13], [1, 1, 1]]):
        s.load(new, 1000 + 100 * i)
        graph.replay()
        s.check()
        torch.cuda.synchronize()
        before = s.out.clone()
        s.out.zero_()
        s.B.tr_paged_decode_attn(s.gs, s.q_out[s.last.long()], s.pages, s.table, s.lens, 50, 3, s.out, s.ws)   # the same, not replayed
        assert torch.equal(before, s.out)


def test_documents_reach_the_pages(B):
    """Assembled rows copied into pages, and stored chunk rows turned into them by their offsets; decode over the pages is decode
    over the contiguous cache."""
    hq, hk, d, page = 8, 2, 128, 16
    gs = B.make_shape(hq, hk, d, "bf16", 1e6)
    lens = [70, 33, 100]
    start = np.concatenate([[0], np.cumsum(lens)])
    n_doc = int(start[-1])
    k, v = (randn(n_doc, hk, d, seed=s, dtype=torch.bfloat16).cuda() for s in (1, 2))
    store = B.Store(gs, k, v, start)
    offsets, _ = B.tr_plan(store, [2, 0, 1], B.TR_POS_REORDERED)
    ck, cv = torch.zeros(n_doc + 1, hk, d, dtype=torch.bfloat16, device="cuda"), torch.zeros(n_doc + 1, hk, d, dtype=torch.bfloat16, device="cuda")
    B.tr_kv_assemble(store, [2, 0, 1], offsets, B.TR_POS_REORDERED, ck, cv)
    q, k1, v1 = (randn(1, h, d, seed=9 + h, dtype=torch.bfloat16).cuda() for h in (hq, hk, hk))
    pos = ints([n_doc])
    B.tr_kv_append(gs, k1, v1, pos, ck, cv, n_doc)
    kv = np.array([0, n_doc + 1])
    want = torch.empty_like(q)
    B.tr_decode_attn(gs, q, ck, cv, pos, kv, want, B.workspace(B.tr_decode_attn_workspace_size(gs, kv)))

    n_blocks = -(-(n_doc + 1) // page)
    table = torch.randperm(n_blocks, generator=torch.Generator().manual_seed(3)).to(torch.int32).cuda().view(1, -1)
    slots = (table[0].repeat_interleave(page) * page + torch.arange(page, device="cuda", dtype=torch.int32).repeat(n_blocks))[:n_doc + 1].contiguous()
    outs = []
    for copy in (True, False):
        kp, vp = (torch.full((n_blocks, page, hk, d), float("nan"), dtype=torch.bfloat16, device="cuda") for _ in range(2))
        pages = B.make_pages(kp, vp)
        if copy:
            B.tr_paged_append(gs, B.tr_rotary_init(0, 0, 1e6), None, ck[:n_doc], cv[:n_doc], None, None, EPS, None, slots[:n_doc], None, pages)
            assert torch.equal(kp.view(-1, hk, d)[slots[:n_doc].long()], ck[:n_doc])
        else:
            for i, c in enumerate([2, 0, 1]):
                at = int(offsets[i])
                turn = torch.full((lens[c],), at, dtype=torch.int32, device="cuda")
                B.tr_paged_append(gs, None, None, k[start[c]:start[c + 1]], v[start[c]:start[c + 1]], None, None, EPS, turn,
                                  slots[at:at + lens[c]], None, pages)
        q_out, out = torch.empty_like(q), torch.empty_like(q)
        B.tr_paged_append(gs, None, q, k1, v1, None, None, EPS, pos, slots[n_doc:], q_out, pages)
        B.tr_paged_decode_attn(gs, q_out, pages, table, ints([n_doc + 1]), 0, 0, out, B.workspace(B.tr_paged_decode_attn_workspace_size(gs, 1, n_blocks, page)))
        outs.append(out)
    # both attentions are within 2e-2 of fp64 over what they read, and what they read differs by single roundings
    for out in outs:
        assert (out.double() - want.double()).abs().max() <= 2 * H.BF16_TOL
