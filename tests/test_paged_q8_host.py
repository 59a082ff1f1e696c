"""Host side of the paged cache in 8 bits, no GPU needed: no-ops, refusals and limits.  Device pointers are made-up addresses: every call fails
validation or is a documented no-op."""
import ctypes as C
import re

import pytest
import torch

from paper_2410_07590_amd import binding as B
from tests.test_paged_host import FAKE, HEADER, fake, p, rotary, shape

SCALES = 100 * 4     # bytes of the scales below


@pytest.fixture(scope="module")
def L():
    return B.lib()


def pages(**kw):
    f = dict(k=FAKE[10], v=FAKE[11], k_scale=FAKE[12] + 3, v_scale=FAKE[13] + 1, page_stride=16 * 512, row_stride=512, head_stride=128, n_pages=100,
             page_size=16, n_kv_heads=4, head_dim=128, reserved=0)
    f.update(kw)
    return B.tr_pages_q8(**f)


def test_the_structure_matches_the_header():
    body = re.search(r"typedef struct tr_pages_q8 \{(.*?)\}", open(HEADER).read(), re.S).group(1)
    names = [d.split()[-1].lstrip("*") for d in re.sub(r"/\*.*?\*/", "", body, flags=re.S).split(";") if d.strip()]
    assert names == [f[0] for f in B.tr_pages_q8._fields_] and C.sizeof(B.tr_pages_q8) == 80


BAD_POOLS = [
    (dict(head_dim=64), B.TR_ERR_SHAPE), (dict(n_kv_heads=2), B.TR_ERR_SHAPE), (dict(reserved=1), -1), (dict(k=0), -1), (dict(v=0), -1), (dict(k_scale=0), -1),
    (dict(v_scale=0), -1), (dict(page_size=8), -1), (dict(page_size=24), -1), (dict(page_size=2048), -1), (dict(page_size=0), -1), (dict(n_pages=0), -1),
    (dict(n_pages=2 ** 27), -1), (dict(k=FAKE[10] + 8), -1), (dict(v=FAKE[11] + 4), -1), (dict(row_stride=520), -1), (dict(row_stride=64), -1),
    (dict(head_stride=0), -1), (dict(head_stride=72), -1), (dict(page_stride=-8192), -1), (dict(page_stride=8200), -1),
    (dict(page_stride=2 ** 32), B.TR_ERR_UNSUPPORTED), (dict(row_stride=2 ** 26 + 16), B.TR_ERR_UNSUPPORTED), (dict(head_stride=2 ** 26 + 16), B.TR_ERR_UNSUPPORTED)]


# ---- append ---------------------------------------------------------------------------------------------------------------------

APP = dict(shape=None, rotary=None, q=FAKE[0], qs=28 * 128, k=FAKE[1], ks=512, v=FAKE[2], vs=512, qn=FAKE[3], kn=FAKE[4], eps=1e-6, pos=FAKE[5],
           slots=FAKE[6], n=9, out=FAKE[7], pages=None)


def append(L, **kw):
    a = dict(APP, **kw)
    sh = a["shape"] or shape()
    pg = a["pages"] or pages()
    i64 = C.c_int64
    return L.tr_paged_append_q8(C.byref(sh), C.byref(a["rotary"]) if a["rotary"] else None, p(a["q"]), i64(a["qs"]), p(a["k"]), i64(a["ks"]), p(a["v"]),
                                i64(a["vs"]), p(a["qn"]), p(a["kn"]), C.c_double(a["eps"]), p(a["pos"]), p(a["slots"]), C.c_int32(a["n"]), p(a["out"]),
                                None if pg == "none" else C.byref(pg), None)


@pytest.mark.parametrize("kw,code", [(dict(pages=pages(**kw)), code) for kw, code in BAD_POOLS] + [
    (dict(shape=shape(d=96)), B.TR_ERR_SHAPE), (dict(rotary=rotary(rotary_dim=144)), B.TR_ERR_SHAPE), (dict(rotary=rotary(freq=1.5)), -1),
    (dict(n=-1), -1), (dict(out=0), -1), (dict(q=0), -1), (dict(k=0), -1), (dict(v=0), -1), (dict(slots=0), -1), (dict(pages="none"), -1), (dict(pos=0), -1),
    (dict(eps=0.0), -1), (dict(k=FAKE[1] + 8), -1), (dict(vs=516), -1), (dict(ks=-512), -1), (dict(out=FAKE[0] + 256), -1),
    # rows that share bytes; codes, scales, inputs and results that do
    (dict(pages=pages(v=FAKE[10])), -1), (dict(pages=pages(row_stride=128)), -1), (dict(pages=pages(page_stride=4096)), -1),
    (dict(pages=pages(k_scale=FAKE[13])), -1), (dict(pages=pages(k_scale=FAKE[13] + 2 - SCALES)), -1), (dict(pages=pages(v_scale=FAKE[10] + 50)), -1),
    (dict(pages=pages(k_scale=FAKE[11] + 99 * 8192 + 16 * 512 - 1)), -1), (dict(pages=pages(k_scale=FAKE[1] + 9 * 1024 - 1)), -1),
    (dict(pages=pages(v_scale=FAKE[6] + 35)), -1), (dict(pages=pages(v_scale=FAKE[5] - SCALES + 1)), -1), (dict(pages=pages(k_scale=FAKE[7])), -1),
    (dict(pages=pages(k_scale=FAKE[0] + 100)), -1), (dict(pages=pages(k_scale=FAKE[4] + 255)), -1), (dict(k=FAKE[10] + 1024), -1), (dict(out=FAKE[11]), -1),
    (dict(shape=shape(hq=2 ** 20 + 1, hkv=2 ** 20 + 1), pages=pages(n_kv_heads=2 ** 20 + 1)), B.TR_ERR_UNSUPPORTED)])
def test_append_refusals(L, kw, code):
    assert append(L, **kw) == code and L.tr_last_error()


def test_append_of_nothing(L):
    assert append(L, n=0) == B.TR_OK
    assert append(L, n=0, pages=pages(k_scale=FAKE[12])) == B.TR_OK
    assert append(L, n=0, q=0, out=0, k=0, v=0, slots=0, pages="none") == B.TR_OK
    assert append(L, q=0, out=0, k=0, v=0, slots=0, pages="none") == B.TR_OK


# ---- read -----------------------------------------------------------------------------------------------------------------------

READ = dict(shape=None, pages=None, table=FAKE[0], blocks=40, lens=FAKE[1], start=FAKE[2], n=6, out_k=FAKE[3], out_v=FAKE[4], rows=1000)


def read(L, **kw):
    a = dict(READ, **kw)
    sh = a["shape"] or shape()
    pg = a["pages"] or pages()
    i = C.c_int32
    return L.tr_paged_read_q8(C.byref(sh), None if pg == "none" else C.byref(pg), p(a["table"]), i(a["blocks"]), p(a["lens"]), p(a["start"]), i(a["n"]),
                              p(a["out_k"]), p(a["out_v"]), i(a["rows"]), None)


@pytest.mark.parametrize("kw,code", [(dict(pages=pages(**kw)), code) for kw, code in BAD_POOLS] + [
    (dict(shape=shape(d=32)), B.TR_ERR_SHAPE), (dict(pages="none"), -1), (dict(n=-1), -1), (dict(blocks=-1), -1), (dict(rows=-1), -1), (dict(table=0), -1),
    (dict(lens=0), -1), (dict(start=0), -1), (dict(out_k=0), -1), (dict(out_v=0), -1), (dict(out_k=FAKE[3] + 8), -1), (dict(out_v=FAKE[4] + 2), -1),
    (dict(n=65537), B.TR_ERR_UNSUPPORTED), (dict(blocks=2 ** 26 + 1), -1), (dict(out_v=FAKE[3]), -1), (dict(out_v=FAKE[3] + 1000 * 1024 - 16), -1),
    (dict(out_k=FAKE[10] + 16), -1), (dict(out_v=FAKE[11] - 16), -1), (dict(out_k=FAKE[12]), -1), (dict(out_v=FAKE[13] - 512000), -1),
    (dict(out_k=FAKE[0] + 944), -1), (dict(out_v=FAKE[1] + 16), -1), (dict(out_k=FAKE[2] + 16), -1),
    (dict(shape=shape(hq=2 ** 20 + 1, hkv=2 ** 20 + 1), pages=pages(n_kv_heads=2 ** 20 + 1)), B.TR_ERR_UNSUPPORTED)])
def test_read_refusals(L, kw, code):
    assert read(L, **kw) == code and L.tr_last_error()


def test_read_of_nothing(L):
    for kw in (dict(n=0), dict(rows=0), dict(blocks=0)):
        assert read(L, **kw) == B.TR_OK
        assert read(L, **kw, table=0, lens=0, start=0, out_k=0, out_v=0) == B.TR_OK


# ---- attention ------------------------------------------------------------------------------------------------------------------

DEC = dict(shape=None, q=FAKE[0], pages=None, table=FAKE[1], blocks=40, lens=FAKE[2], n=6, window=0, sinks=0, out=FAKE[3], ws=FAKE[4], bytes=1 << 31)


def decode(L, **kw):
    a = dict(DEC, **kw)
    sh = a["shape"] or shape()
    pg = a["pages"] or pages()
    i = C.c_int32
    return L.tr_paged_decode_attn_q8(C.byref(sh), p(a["q"]), None if pg == "none" else C.byref(pg), p(a["table"]), i(a["blocks"]), p(a["lens"]), i(a["n"]),
                                     i(a["window"]), i(a["sinks"]), p(a["out"]), p(a["ws"]), C.c_size_t(a["bytes"]), None)


@pytest.mark.parametrize("kw,code", [(dict(pages=pages(**kw)), code) for kw, code in BAD_POOLS] + [
    (dict(shape=shape(d=32)), B.TR_ERR_SHAPE), (dict(pages="none"), -1), (dict(q=0), -1), (dict(table=0), -1), (dict(lens=0), -1), (dict(out=0), -1),
    (dict(n=-1), -1), (dict(blocks=-1), -1), (dict(window=-1), -1), (dict(sinks=-1), -1), (dict(q=FAKE[0] + 4), -1), (dict(out=FAKE[3] + 8), -1),
    (dict(blocks=2 ** 28), -1), (dict(out=FAKE[0] + 256), -1), (dict(out=FAKE[1] + 16), -1), (dict(out=FAKE[2]), -1), (dict(out=FAKE[10]), -1),
    (dict(out=FAKE[11] + 4096), -1), (dict(out=FAKE[12]), -1), (dict(out=FAKE[13] + 16 * 25), -1),
    (dict(ws=0), B.TR_ERR_WORKSPACE), (dict(ws=FAKE[4] + 16), B.TR_ERR_WORKSPACE), (dict(bytes=1000), B.TR_ERR_WORKSPACE),
    (dict(n=65537), B.TR_ERR_UNSUPPORTED), (dict(n=4096, blocks=2 ** 19), B.TR_ERR_UNSUPPORTED),
    (dict(n=60000, shape=shape(hq=1024, hkv=512), pages=pages(n_kv_heads=512, row_stride=512 * 128, page_stride=2 ** 20)), B.TR_ERR_UNSUPPORTED)])
def test_decode_refusals(L, kw, code):
    assert decode(L, **kw) == code and L.tr_last_error()


def test_decode_of_nothing(L):
    assert decode(L, n=0) == B.TR_OK
    assert decode(L, n=0, q=0, table=0, lens=0, out=0, ws=0, bytes=0) == B.TR_OK


def test_workspaces_at_both_sides_of_the_limits(L):
    size = B.tr_paged_decode_attn_q8_workspace_size
    most = 2 ** 31 - 1
    for args in ((shape(d=96), 4, 9, 16), (shape(), 0, 9, 16), (shape(), -4, 9, 16), (shape(), 4, 0, 16), (shape(), 4, 9, 8), (shape(), 4, 9, 24), (shape(), 65537, 1, 16),
                 (shape(hq=most, hkv=most), most, most, 1024), (shape(hq=4096, hkv=4097), 4, 9, 16), (shape(hq=4096, hkv=4096), 4097, 9, 16),
                 (shape(), 1, 2 ** 20 + 1, 1024), (shape(hq=4, hkv=4), 4096, 2 ** 18 + 1, 16)):
        assert size(*args) == 0, args[1:]
    # a unit is 64 keys whatever the type: 2^30 of them are 4 heads x 4096 requests x 2^18 pages of 16
    for dtype in (B.TR_BF16, B.TR_F32):
        assert size(shape(hq=4, hkv=4, dtype=dtype), 4096, 2 ** 18, 16) > 0
        assert size(shape(dtype=dtype), 65536, 9, 16) > 0 and size(shape(dtype=dtype), 1, 2 ** 20, 1024) > 0
    assert size(shape(), 100, 4, 16) == 0 and size(shape(), 100, 5, 16) > 0   # a unit is never cut
    need = size(shape(), 6, 40, 16)
    assert decode(L, bytes=need - 1) == B.TR_ERR_WORKSPACE


# ---- the binding ----------------------------------------------------------------------------------------------------------------

def test_binding_refuses_wrong_types_and_sizes(L):
    bf, sh = torch.bfloat16, shape(4, 2, 64)
    pg = pages(n_kv_heads=2, head_dim=64, head_stride=64)
    ok = dict(shape=sh, rotary=None, q=fake(5, 4, 64, dtype=bf), k=fake(5, 2, 64, dtype=bf), v=fake(5, 2, 64, dtype=bf), q_norm=None, k_norm=None, eps=1e-6,
              pos=fake(5), slots=fake(5), q_out=fake(5, 4, 64, dtype=bf), pages=pg, stream=0)
    for kw in (dict(q=fake(5, 4, 64)), dict(k=fake(5, 3, 64, dtype=bf)), dict(v=fake(4, 2, 64, dtype=bf)), dict(slots=fake(6)), dict(k_norm=fake(32, dtype=bf))):
        with pytest.raises(AssertionError):
            B.tr_paged_append_q8(**dict(ok, **kw))
    with pytest.raises(TypeError):
        B.tr_paged_append_q8(**dict(ok, pages=B.tr_pages()))
    ok = dict(shape=sh, pages=pg, block_table=fake(3, 7), kv_lens=fake(3), row_start=fake(4), out_k=fake(9, 2, 64, dtype=bf), out_v=fake(9, 2, 64, dtype=bf), stream=0)
    for kw in (dict(out_k=fake(9, 2, 64, dtype=torch.float32)), dict(out_v=fake(8, 2, 64, dtype=bf)), dict(out_k=fake(9, 128, dtype=bf)), dict(row_start=fake(3)),
               dict(kv_lens=fake(2)), dict(block_table=fake(21)), dict(row_start=fake(4, dtype=torch.int64)), dict(out_v=fake(9, 4, 64, dtype=bf)[:, ::2])):
        with pytest.raises(AssertionError):
            B.tr_paged_read_q8(**dict(ok, **kw))
    ok = dict(shape=sh, q=fake(3, 4, 64, dtype=bf), pages=pg, block_table=fake(3, 7), kv_lens=fake(3), window=0, n_sink=0, out=fake(3, 4, 64, dtype=bf),
              workspace=None, stream=0)
    for kw in (dict(q=fake(3, 4, 64, dtype=torch.float32)), dict(q=fake(2, 4, 64, dtype=bf)), dict(block_table=fake(4, 7)), dict(kv_lens=fake(2))):
        with pytest.raises(AssertionError):
            B.tr_paged_decode_attn_q8(**dict(ok, **kw))
    with pytest.raises(TypeError):
        B.tr_paged_decode_attn_q8(**dict(ok, pages=B.tr_pages()))


def test_pools_of_tensors_that_do_not_fit_each_other(L):
    e4, e8 = torch.float8_e4m3fn, torch.float8_e8m0fnu
    ok = dict(k_pages=fake(5, 32, 2, 64, dtype=e4), v_pages=fake(5, 32, 2, 64, dtype=e4), k_scale=fake(5, 2, 2, dtype=e8), v_scale=fake(5, 2, 2, dtype=torch.uint8))
    for kw in (dict(k_pages=fake(5, 32, 2, 64, dtype=torch.uint8)), dict(k_pages=fake(5, 32, 2, 64, dtype=torch.bfloat16), v_pages=fake(5, 32, 2, 64, dtype=torch.bfloat16)),
               dict(v_pages=fake(4, 32, 2, 64, dtype=e4)), dict(k_scale=fake(5, 2, 2, dtype=e4)), dict(k_scale=fake(5, 2, dtype=e8)), dict(v_scale=fake(5, 1, 2, dtype=e8)),
               dict(v_scale=fake(5, 4, 2, dtype=e8)[:, ::2]), dict(k_scale=torch.zeros(5, 2, 2, dtype=torch.uint8))):
        with pytest.raises(AssertionError):
            B.make_pages_q8(**dict(ok, **kw))
