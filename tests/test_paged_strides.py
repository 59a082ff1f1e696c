"""Which pools tr_paged_append takes, no GPU needed: every row of K and of V has bytes of its own, or the call is refused.  Against sets of
bytes written out.  An accepted call would launch, so all calls carry a misaligned k, which is refused last and by a message of its own."""
import ctypes as C

import numpy as np
import pytest

from paper_2410_07590_amd import binding as B

K_AT = 0x7000_0000_0000
AT = [0x7100_0000_0000 + (i << 36) for i in range(8)]


@pytest.fixture(scope="module")
def L():
    return B.lib()


def accepted(L, dtype, d, heads, n_pages, page, page_stride, row_stride, head_stride, v_from_k):
    """Strides and the distance of V from K in elements."""
    e = 4 if dtype == B.TR_F32 else 2
    sh = B.tr_shape(heads, heads, d, dtype, 1e4, 0, 0)
    pg = B.tr_pages(K_AT, K_AT + v_from_k * e, page_stride, row_stride, head_stride, n_pages, page, heads, d, dtype, 0)
    p, i64 = C.c_void_p, C.c_int64
    rc = L.tr_paged_append(C.byref(sh), None, None, i64(0), p(AT[0] + 8), i64(heads * d), p(AT[1]), i64(heads * d), None, None, C.c_double(1e-6),
                           p(AT[2]), p(AT[3]), C.c_int32(1), None, C.byref(pg), None)
    assert rc == B.TR_ERR_INVALID_ARG
    text = L.tr_last_error().decode()
    assert "16-byte aligned" in text or "same bytes" in text, text
    return "same bytes" not in text


def bytes_are_its_own(d, heads, n_pages, page, page_stride, row_stride, head_stride, v_from_k):
    at = (np.arange(n_pages)[:, None, None, None] * page_stride + np.arange(page)[:, None, None] * row_stride + np.arange(heads)[:, None] * head_stride +
          np.arange(0, d, 8)).ravel()   # pieces of 8 elements: strides and distances are multiples of that
    both = np.concatenate([at, at + v_from_k])
    return len(np.unique(both)) == len(both)


@pytest.mark.parametrize("what,heads,n_pages,page,strides,v", [
    ("a head is its neighbour's row", 4, 8, 16, (16 * 512, 128, 128), 1 << 24), ("a page is its neighbour's row", 4, 8, 16, (512, 512, 128), 1 << 24),
    ("V is K a row later", 4, 8, 16, (16 * 512, 512, 128), 512), ("V is K a head later", 4, 8, 16, (16 * 512, 512, 128), 128),
    ("V is K half a head later", 4, 8, 16, (16 * 512, 512, 128), 64), ("V is K a page later", 4, 8, 16, (16 * 512, 512, 128), 16 * 512),
    ("V is K a row sooner", 4, 8, 16, (16 * 512, 512, 128), -512), ("rows reach into each other", 4, 8, 16, (16 * 512, 448, 128), 1 << 24),
    ("V is K", 4, 8, 16, (16 * 512, 512, 128), 0), ("pages reach into each other, one head", 1, 8, 16, (15 * 128, 128, 0), 1 << 24)])
def test_pools_that_use_bytes_twice(L, what, heads, n_pages, page, strides, v):
    assert not accepted(L, B.TR_BF16, 128, heads, n_pages, page, *strides, v), what


@pytest.mark.parametrize("what,heads,n_pages,page,strides,v", [
    ("rows", 4, 8, 16, (16 * 512, 512, 128), 8 * 16 * 512), ("V in front", 4, 8, 16, (16 * 512, 512, 128), -8 * 16 * 512),
    ("heads", 4, 8, 16, (16 * 512, 128, 16 * 128), 8 * 16 * 512), ("K and V of a page together", 4, 8, 16, (2 * 16 * 512, 512, 128), 16 * 512),
    ("V of a page first", 4, 8, 16, (2 * 16 * 512, 512, 128), -16 * 512), ("K and V of a row together", 4, 8, 16, (16 * 1024, 1024, 128), 512),
    ("K and V of a head together", 4, 8, 16, (16 * 1024, 1024, 256), 128), ("padding", 4, 8, 16, (20 * 800, 800, 144), 1 << 24),
    ("V in the padding of K's rows", 4, 8, 16, (16 * 1100 * 8, 1100 * 8, 144), 4 * 144), ("a page with a stride of nothing", 4, 1, 16, (0, 512, 128), 16 * 512),
    ("a head with a stride of nothing", 1, 8, 16, (16 * 128, 128, 0), 8 * 16 * 128), ("rows outside of pages", 4, 8, 16, (512, 8 * 512, 128), 8 * 16 * 512),
    ("more than 4 GiB", 8, 1 << 20, 16, (2 * 16 * 1024, 1024, 128), 16 * 1024)])
def test_pools_whose_rows_are_apart(L, what, heads, n_pages, page, strides, v):
    assert accepted(L, B.TR_BF16, 128, heads, n_pages, page, *strides, v), what


def test_pools_of_any_strides_against_their_bytes(L):
    rng = np.random.default_rng(7)
    seen = [0, 0]
    for _ in range(6000):
        d, heads, n_pages, page = 64, int(rng.integers(1, 5)), int(rng.integers(1, 5)), 8
        sizes = [64, 64, 72, 128, 192, 256, 512, 64 * heads, 64 * page, 64 * heads * page, 128 * heads * page, 8 * int(rng.integers(8, 600))]
        head, row, pages = (int(rng.choice(sizes)) * int(rng.choice([1, 1, 1, 2])) for _ in range(3))
        if rng.random() < 0.5:
            head, row, pages = sorted((head, row, pages))
            if rng.random() < 0.3:
                head, row = row, head
        v = int(rng.choice([1, -1])) * int(rng.choice([64, head, row, pages, heads * head, page * row, n_pages * pages, 2 * pages, 8 * int(rng.integers(0, 4000)), 1 << 22]))
        want = bytes_are_its_own(d, heads, n_pages, page, pages, row, head, v)
        got = accepted(L, B.TR_BF16, d, heads, n_pages, page, pages, row, head, v)
        # strides that interleave (a stride below the extent of what lies inside it) may keep rows apart all the same and are refused
        nested, extent = True, d
        for stride, count in sorted((s, c) for s, c in ((head, heads), (row, page), (pages, n_pages)) if c > 1):
            nested &= stride >= extent
            extent += (count - 1) * stride
        assert got == (want and nested), (heads, n_pages, pages, row, head, v, want, nested)
        seen[got] += 1
    assert min(seen) > 500, seen
