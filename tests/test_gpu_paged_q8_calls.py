"""Calls over a paged cache in 8 bits that the interface allows: queries in place, keys and values in one allocation, scales at odd addresses."""
import numpy as np
import pytest
import torch

from tests import paged_q8_reference as Q
from tests import paged_reference as R
from tests.test_gpu_paged import DT, ints, randn, tables
from tests.test_gpu_paged_q8 import EPS

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2410_07590_amd import binding
    binding.lib()
    return binding


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("n", [1, 7, 5001])
@pytest.mark.parametrize("d,layout,rot", [(64, 0, 32), (128, 1, 128)])
def test_queries_in_place(B, dt, n, d, layout, rot):
    """Bit for bit what they are elsewhere, beside keys and values of their own.  One token's queries may lie in a packed projection."""
    hq, hk = 9, 3
    qkv = randn(n, hq + 2 * hk, d, seed=n, dtype=DT[dt]).cuda()
    q, k, v = (qkv[:, :hq], qkv[:, hq:hq + hk], qkv[:, hq + hk:]) if n == 1 else (qkv[:, :hq].contiguous(), qkv[:, hq:hq + hk], qkv[:, hq + hk:])
    w, pos, slots = randn(d, seed=1, dtype=DT[dt]).cuda(), ints(np.arange(n) * 3), ints(np.arange(n) + 5)
    gs, rotary = B.make_shape(hq, hk, d, dt, 1e4, layout), B.tr_rotary_init(layout, rot, 1e4)

    def append(out):
        codes = [torch.zeros(-(-(n + 5) // 32), 32, hk, d, dtype=torch.uint8, device="cuda") for _ in range(2)]
        scales = [torch.full((len(codes[0]), hk, 2), 127, dtype=torch.uint8, device="cuda") for _ in range(2)]
        B.tr_paged_append_q8(gs, rotary, q, k, v, w, w, EPS, pos, slots, out, B.make_pages_q8(*codes, *scales))
        torch.cuda.synchronize()
        return codes + scales

    out = torch.empty(n, hq, d, dtype=DT[dt], device="cuda")
    want = append(out)
    got = append(q)
    assert torch.equal(q, out) and all(torch.equal(a, b) for a, b in zip(want, got))


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("hk,d,form", [(2, 128, "page, side, row, head"), (3, 64, "page, row, side, head"), (2, 64, "page, row, head, side"), (4, 64, "side, page, head, row")])
def test_keys_and_values_in_one_allocation_with_scales_at_odd_addresses(B, dt, hk, d, form):
    """Append, read back and decode; the byte in front of each array of scales and the one behind it stay."""
    page, lens, hq = 32, [75, 1, 40, 32], 2 * hk
    table, n_pages = tables(np.random.default_rng(d), lens, page)
    shape = {"page": n_pages, "side": 2, "row": page, "head": hk}
    names = form.split(", ")
    whole = torch.zeros([shape[x] for x in names] + [d], dtype=torch.uint8, device="cuda")
    kp, vp = (whole.permute(*(names.index(x) for x in ("side", "page", "row", "head")), 4)[i] for i in (0, 1))
    room = [torch.full((n_pages * hk * 2 + 2,), 127, dtype=torch.uint8, device="cuda") for _ in range(2)]
    ks, vs = (r[1:-1].view(n_pages, hk, 2) for r in room)
    assert ks.data_ptr() % 2 == 1
    pages, gs = B.make_pages_q8(kp, vp, ks, vs), B.make_shape(hq, hk, d, dt, 1e4)
    slots = np.concatenate([table[r, np.arange(n) // page] * page + np.arange(n) % page for r, n in enumerate(lens)])
    k, v = (randn(len(slots), hk, d, seed=i, dtype=DT[dt]) for i in (1, 2))
    B.tr_paged_append_q8(gs, B.tr_rotary_init(0, 0, 1e4), None, k.cuda(), v.cuda(), None, None, EPS, None, ints(slots), None, pages)
    torch.cuda.synchronize()
    held = [(kp.cpu(), ks.cpu()), (vp.cpu(), vs.cpu())]
    for (codes, scale), x in zip(held, (k, v)):
        Q.check_append(codes, scale, torch.zeros_like(codes), torch.full_like(scale, 127), x.double(), 0, slots, form)
    assert all(int(r[0]) == 127 and int(r[-1]) == 127 for r in room)
    starts = np.concatenate([[0], np.cumsum(lens)])
    rows = [torch.empty(len(slots), hk, d, dtype=DT[dt], device="cuda") for _ in range(2)]
    B.tr_paged_read_q8(gs, pages, ints(table), ints(lens), ints(starts), *rows)
    q = randn(len(lens), hq, d, seed=5, dtype=DT[dt])
    out = torch.empty_like(q).cuda()
    B.tr_paged_decode_attn_q8(gs, q.cuda(), pages, ints(table), ints(lens), 0, 0, out,
                              B.workspace(B.tr_paged_decode_attn_q8_workspace_size(gs, len(lens), table.shape[1], page)))
    torch.cuda.synchronize()
    worth = [Q.values(*h) for h in held]
    for got, w in zip(rows, worth):
        assert torch.equal(got.cpu().double(), w.reshape(-1, hk, d)[torch.from_numpy(slots)])
    want, bound = R.decode_batch(q, *worth, torch.from_numpy(table), lens, 0, 0, 2)
    R.assert_within(out, want, torch.finfo(DT[dt]).eps / 2 * want.abs() * 1.01 + bound, form)
