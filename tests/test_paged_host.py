"""Host side of the paged cache, no GPU needed: frequencies, no-ops and refusals.  Device pointers are made-up addresses: every
call fails validation or is a documented no-op."""
import ctypes as C
import math
import os
import re

import numpy as np
import pytest
import torch

from paper_2410_07590_amd import binding as B
from tests import paged_reference as R

HEADER = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "turborag.h")
FAKE = [0x7000_0000_0000 + (i << 32) for i in range(16)]   # 4 GiB apart


@pytest.fixture(scope="module")
def L():
    return B.lib()


def p(a):
    return C.c_void_p(a)


def shape(hq=28, hkv=4, d=128, dtype=B.TR_BF16, base=1e6, layout=0):
    return B.tr_shape(hq, hkv, d, dtype, float(base), layout, 0)


def pages(**kw):
    f = dict(k=FAKE[10], v=FAKE[11], page_stride=16 * 512, row_stride=512, head_stride=128, n_pages=100, page_size=16, n_kv_heads=4, head_dim=128,
             dtype=B.TR_BF16, reserved=0)
    f.update(kw)
    return B.tr_pages(**f)


def test_enumerators_and_structures_match_the_header():
    text = open(HEADER).read()
    for name in ("TR_SCALE_NONE", "TR_SCALE_LINEAR", "TR_SCALE_BASE", "TR_SCALE_PARTS"):
        assert getattr(B, name) == int(re.search(r"\b%s\s*=\s*(\d+)" % name, text).group(1))
    for cls in (B.tr_pages, B.tr_rotary):
        body = re.sub(r"/\*.*?\*/", "", re.search(r"typedef struct %s \{(.*?)\}" % cls.__name__, text, re.S).group(1), flags=re.S)
        names = [re.sub(r"\[.*", "", d.split()[-1]).lstrip("*") for d in body.split(";") if d.strip()]
        assert names == [f[0] for f in cls._fields_]
    assert C.sizeof(B.tr_pages) == 64 and C.sizeof(B.tr_rotary) == 528


# ---- frequencies ----------------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("rot", [16, 32, 64, 112, 128])
@pytest.mark.parametrize("base", [1e4, 1e6])
def test_rotary_frequencies(L, rot, base):
    for scaling, code in (("none", 0), ("linear", 1), ("base", 2), ("parts", 3)):
        for factor in (1.0, 2.5, 16.0):
            r = B.tr_rotary_init(1, rot, base, code, factor, 8192, 1.0, 32.0, 1.25)
            want = R.frequencies(rot, base, scaling, factor, 8192)
            assert r.layout == 1 and r.rotary_dim == rot and r.amplitude == 1.25
            # a power of b, its exponent off by a few steps of its size, is off by ln(b) times them
            assert np.allclose(np.array(r.freq[:rot // 2]), want, rtol=64 * 2.0 ** -53 * math.log(base * factor ** 1.2), atol=0)
            assert all(f == 0 for f in r.freq[rot // 2:])
    assert np.array_equal(B.tr_rotary_init(0, rot, base, B.TR_SCALE_PARTS, 1.0, 8192).freq[:], B.tr_rotary_init(0, rot, base).freq[:])
    stretched = B.tr_rotary_init(0, rot, base, B.TR_SCALE_BASE, 8.0).freq
    plain = B.tr_rotary_init(0, rot, base).freq
    assert stretched[0] == plain[0] == 1.0
    assert abs(stretched[rot // 2 - 1] * 8.0 / plain[rot // 2 - 1] - 1) < 1e-12
    parts = B.tr_rotary_init(0, rot, base, B.TR_SCALE_PARTS, 4.0, 4096, 1.0, 32.0).freq
    for m in range(rot // 2):
        turns = 4096 * plain[m] / (2 * math.pi)
        assert parts[m] == plain[m] if turns >= 32 else parts[m] < plain[m]
        if turns <= 1:
            assert parts[m] == plain[m] / 4.0


def test_rotary_without_channels():
    r = B.tr_rotary_init(0, 0, 1e4, B.TR_SCALE_BASE, 4.0)
    assert r.rotary_dim == 0 and all(f == 0 for f in r.freq)


@pytest.mark.parametrize("args,code", [
    ((2, 64, 1e4, 0, 1, 0, 1, 32, 1), B.TR_ERR_INVALID_ARG), ((0, 24, 1e4, 0, 1, 0, 1, 32, 1), B.TR_ERR_SHAPE),
    ((0, 144, 1e4, 0, 1, 0, 1, 32, 1), B.TR_ERR_SHAPE), ((0, -16, 1e4, 0, 1, 0, 1, 32, 1), B.TR_ERR_SHAPE),
    ((0, 64, 1.0, 0, 1, 0, 1, 32, 1), B.TR_ERR_INVALID_ARG), ((0, 64, math.inf, 0, 1, 0, 1, 32, 1), B.TR_ERR_INVALID_ARG),
    ((0, 64, math.nan, 0, 1, 0, 1, 32, 1), B.TR_ERR_INVALID_ARG), ((0, 64, 1e4, 4, 1, 0, 1, 32, 1), B.TR_ERR_INVALID_ARG),
    ((0, 64, 1e4, 1, 0.5, 0, 1, 32, 1), B.TR_ERR_INVALID_ARG), ((0, 64, 1e4, 2, math.nan, 0, 1, 32, 1), B.TR_ERR_INVALID_ARG),
    ((0, 64, 1e4, 2, 1e308, 0, 1, 32, 1), B.TR_ERR_INVALID_ARG), ((0, 64, 1e4, 3, 2, 0, 1, 32, 1), B.TR_ERR_INVALID_ARG),
    ((0, 64, 1e4, 3, 2, 4096, 32, 32, 1), B.TR_ERR_INVALID_ARG), ((0, 64, 1e4, 3, 2, 4096, 1, math.inf, 1), B.TR_ERR_INVALID_ARG),
    ((0, 64, 1e4, 0, 1, 0, 1, 32, math.nan), B.TR_ERR_INVALID_ARG)])
def test_rotary_refusals(args, code):
    with pytest.raises(B.TurboRagError) as e:
        B.tr_rotary_init(*args)
    assert e.value.code == code


# ---- block tables ---------------------------------------------------------------------------------------------------------------

MAP = dict(cached=FAKE[0], new=FAKE[1], first=FAKE[2], n_req=5, page=16, free=FAKE[3], n_free=10, table=FAKE[4], blocks=7, lens=FAKE[5],
           cu=FAKE[6], slots=FAKE[7], pos=FAKE[8], n_slots=100, counts=FAKE[9])


def page_map(L, **kw):
    a = dict(MAP, **kw)
    i = C.c_int32
    return L.tr_page_map(p(a["cached"]), p(a["new"]), p(a["first"]), i(a["n_req"]), i(a["page"]), p(a["free"]), i(a["n_free"]), p(a["table"]),
                         i(a["blocks"]), p(a["lens"]), p(a["cu"]), p(a["slots"]), p(a["pos"]), i(a["n_slots"]), p(a["counts"]), None)


@pytest.mark.parametrize("kw", [dict(cached=0), dict(new=0), dict(free=0), dict(table=0), dict(lens=0), dict(cu=0), dict(slots=0), dict(pos=0), dict(counts=0),
                                dict(n_req=-1), dict(n_free=-1), dict(blocks=-1), dict(n_slots=-1), dict(page=0), dict(page=24), dict(page=4), dict(page=2048),
                                dict(page=-16), dict(lens=FAKE[0]), dict(lens=FAKE[0] + 16), dict(cu=FAKE[1] - 20), dict(slots=FAKE[8] + 396), dict(pos=FAKE[3] + 36),
                                dict(counts=FAKE[4] + 136), dict(table=FAKE[2] + 16), dict(counts=FAKE[6] + 20)])
def test_map_refusals(L, kw):
    assert page_map(L, **kw) == B.TR_ERR_INVALID_ARG and L.tr_last_error()


def test_map_of_too_many_requests(L):
    assert page_map(L, n_req=4097) == B.TR_ERR_UNSUPPORTED


# ---- append ---------------------------------------------------------------------------------------------------------------------

APP = dict(shape=None, rotary=None, q=FAKE[0], qs=28 * 128, k=FAKE[1], ks=512, v=FAKE[2], vs=512, qn=FAKE[3], kn=FAKE[4], eps=1e-6, pos=FAKE[5],
           slots=FAKE[6], n=9, out=FAKE[7], pages=None)


def append(L, **kw):
    a = dict(APP, **kw)
    sh = a["shape"] or shape()
    pg = a["pages"] or pages()
    i64 = C.c_int64
    return L.tr_paged_append(C.byref(sh), C.byref(a["rotary"]) if a["rotary"] else None, p(a["q"]), i64(a["qs"]), p(a["k"]), i64(a["ks"]), p(a["v"]),
                             i64(a["vs"]), p(a["qn"]), p(a["kn"]), C.c_double(a["eps"]), p(a["pos"]), p(a["slots"]), C.c_int32(a["n"]), p(a["out"]),
                             None if pg == "none" else C.byref(pg), None)


def rotary(**kw):
    r = B.tr_rotary_init(0, 64, 1e4)
    for k, v in kw.items():
        if k == "freq":
            r.freq[5] = v
        else:
            setattr(r, k, v)
    return r


@pytest.mark.parametrize("kw,code", [
    (dict(shape=shape(d=96)), B.TR_ERR_SHAPE), (dict(shape=shape(dtype=B.TR_F32)), B.TR_ERR_SHAPE), (dict(shape=shape(hkv=7)), B.TR_ERR_SHAPE),
    (dict(pages=pages(head_dim=64)), B.TR_ERR_SHAPE), (dict(pages=pages(dtype=0)), B.TR_ERR_SHAPE),
    (dict(rotary=rotary(rotary_dim=144)), B.TR_ERR_SHAPE), (dict(rotary=rotary(rotary_dim=8)), B.TR_ERR_SHAPE),
    (dict(shape=shape(d=64), pages=pages(head_dim=64, row_stride=256, head_stride=64), rotary=B.tr_rotary_init(0, 128, 1e4)), B.TR_ERR_SHAPE),
    (dict(rotary=rotary(layout=2)), -1), (dict(rotary=rotary(amplitude=math.inf)), -1), (dict(rotary=rotary(freq=1.5)), -1),
    (dict(rotary=rotary(freq=-0.1)), -1), (dict(rotary=rotary(freq=math.nan)), -1),
    (dict(n=-1), -1), (dict(out=0), -1), (dict(q=0), -1), (dict(k=0), -1), (dict(v=0), -1), (dict(slots=0), -1), (dict(pages="none"), -1), (dict(pos=0), -1),
    (dict(eps=0.0), -1), (dict(eps=-1.0), -1), (dict(eps=math.nan), -1), (dict(eps=math.inf), -1), (dict(eps=1e-60), -1), (dict(eps=1e300), -1),
    (dict(q=FAKE[0] + 2), -1), (dict(k=FAKE[1] + 8), -1), (dict(v=FAKE[2] + 8), -1), (dict(out=FAKE[7] + 8), -1), (dict(qn=FAKE[3] + 2), -1),
    (dict(kn=FAKE[4] + 2), -1), (dict(qs=28 * 128 + 4), -1), (dict(ks=516), -1), (dict(vs=517), -1), (dict(qs=-3584), -1), (dict(ks=2 ** 62), -1),
    (dict(out=FAKE[5]), -1), (dict(out=FAKE[6] + 16), -1), (dict(out=FAKE[3]), -1), (dict(out=FAKE[4] + 240), -1), (dict(slots=FAKE[11] + 32), -1),
    (dict(out=FAKE[0] + 256), -1), (dict(out=FAKE[0], qs=28 * 128 + 8), -1), (dict(out=FAKE[1]), -1), (dict(out=FAKE[2] + 4096), -1),
    (dict(k=FAKE[10] + 1024), -1), (dict(out=FAKE[11]), -1), (dict(q=FAKE[11] + 99 * 16384 + 15 * 1024 + 768, qs=0), -1),
    (dict(pages=pages(page_size=12)), -1), (dict(pages=pages(page_size=4)), -1), (dict(pages=pages(n_pages=0)), -1), (dict(pages=pages(n_pages=2 ** 27)), -1),
    (dict(pages=pages(reserved=1)), -1), (dict(pages=pages(k=0)), -1), (dict(pages=pages(v=FAKE[11] + 8)), -1), (dict(pages=pages(v=FAKE[10])), -1), (dict(pages=pages(row_stride=64)), -1),
    (dict(pages=pages(row_stride=516)), -1), (dict(pages=pages(head_stride=0)), -1), (dict(pages=pages(page_stride=-8192)), -1),
    (dict(pages=pages(page_stride=2 ** 60)), B.TR_ERR_UNSUPPORTED), (dict(pages=pages(page_stride=2 ** 31)), B.TR_ERR_UNSUPPORTED),
    (dict(pages=pages(row_stride=2 ** 26)), B.TR_ERR_UNSUPPORTED)])
def test_append_refusals(L, kw, code):
    assert append(L, **kw) == code and L.tr_last_error()


def test_append_of_nothing(L):
    assert append(L, n=0) == B.TR_OK
    assert append(L, n=0, q=0, out=0, k=0, v=0, slots=0, pages="none") == B.TR_OK
    assert append(L, q=0, out=0, k=0, v=0, slots=0, pages="none") == B.TR_OK     # neither side


# ---- attention ------------------------------------------------------------------------------------------------------------------

DEC = dict(shape=None, q=FAKE[0], pages=None, table=FAKE[1], blocks=40, lens=FAKE[2], n=6, window=0, sinks=0, out=FAKE[3], ws=FAKE[4], bytes=1 << 31)


def decode(L, **kw):
    a = dict(DEC, **kw)
    sh = a["shape"] or shape()
    pg = a["pages"] or pages()
    i = C.c_int32
    return L.tr_paged_decode_attn(C.byref(sh), p(a["q"]), None if pg == "none" else C.byref(pg), p(a["table"]), i(a["blocks"]), p(a["lens"]), i(a["n"]),
                                  i(a["window"]), i(a["sinks"]), p(a["out"]), p(a["ws"]), C.c_size_t(a["bytes"]), None)


@pytest.mark.parametrize("kw,code", [
    (dict(shape=shape(d=32)), B.TR_ERR_SHAPE), (dict(shape=shape(hkv=2)), B.TR_ERR_SHAPE), (dict(pages=pages(dtype=0)), B.TR_ERR_SHAPE),
    (dict(pages="none"), -1), (dict(q=0), -1), (dict(table=0), -1), (dict(lens=0), -1), (dict(out=0), -1), (dict(n=-1), -1), (dict(blocks=-1), -1),
    (dict(window=-1), -1), (dict(sinks=-1), -1), (dict(q=FAKE[0] + 4), -1), (dict(out=FAKE[3] + 8), -1), (dict(blocks=2 ** 28), -1),
    (dict(pages=pages(page_size=0)), -1), (dict(pages=pages(k=0)), -1), (dict(pages=pages(page_stride=4)), -1),
    (dict(out=FAKE[0] + 256), -1), (dict(out=FAKE[1] + 16), -1), (dict(out=FAKE[2]), -1), (dict(out=FAKE[10]), -1), (dict(out=FAKE[11] + 4096), -1),
    (dict(ws=0), B.TR_ERR_WORKSPACE), (dict(ws=FAKE[4] + 16), B.TR_ERR_WORKSPACE), (dict(bytes=1000), B.TR_ERR_WORKSPACE),
    (dict(n=65537), B.TR_ERR_UNSUPPORTED), (dict(n=4096, blocks=2 ** 18), B.TR_ERR_UNSUPPORTED), (dict(pages=pages(row_stride=2 ** 26)), B.TR_ERR_UNSUPPORTED),
    (dict(n=60000, shape=shape(hq=1024, hkv=512), pages=pages(n_kv_heads=512, row_stride=512 * 128, page_stride=2 ** 20)), B.TR_ERR_UNSUPPORTED)])
def test_decode_refusals(L, kw, code):
    assert decode(L, **kw) == code and L.tr_last_error()


def test_decode_of_nothing(L):
    assert decode(L, n=0) == B.TR_OK
    assert decode(L, n=0, q=0, table=0, lens=0, out=0, ws=0, bytes=0) == B.TR_OK


def test_workspace_queries_that_make_no_sense_are_zero(L):
    for args in ((shape(d=96), 4, 9, 16), (shape(), 0, 9, 16), (shape(), -4, 9, 16), (shape(), 4, 0, 16), (shape(), 4, 9, 15)):
        assert B.tr_paged_decode_attn_workspace_size(*args) == 0


def test_workspace_queries_of_sizes_that_are_refused_are_zero(L):
    most = 2 ** 31 - 1
    for args in ((shape(), 65537, 1, 16), (shape(), most, most, 1024), (shape(hq=most, hkv=most), most, most, 1024), (shape(hq=4096, hkv=4096), 4096, 9, 16),
                 (shape(), 1, 2 ** 20 + 1, 1024), (shape(), 4096, 2 ** 18, 16)):
        assert B.tr_paged_decode_attn_workspace_size(*args) == 0
    assert B.tr_paged_decode_attn_workspace_size(shape(), 65536, 9, 16) > 0
    assert B.tr_paged_decode_attn_workspace_size(shape(), 1, 2 ** 20, 1024) > 0


def test_append_of_too_many_heads(L):
    big = shape(hq=2 ** 20 + 1, hkv=2 ** 20 + 1)
    assert append(L, shape=big, pages=pages(n_kv_heads=2 ** 20 + 1)) == B.TR_ERR_UNSUPPORTED


# ---- the binding ------------------------------------------------------------------------------------------------------------------

def fake(*size, dtype=torch.int32):
    from torch._subclasses.fake_tensor import FakeTensorMode
    with FakeTensorMode():
        return torch.empty(*size, dtype=dtype, device="cuda")


def test_binding_refuses_wrong_types_and_sizes(L):
    ok = dict(cached_lens=fake(3), new_lens=fake(3), first_pos=None, page_size=16, free_pages=fake(9), block_table=fake(3, 4), kv_lens=fake(3),
              cu_new=fake(4), slots=fake(10), pos=fake(10), counts=fake(2), stream=0)
    for kw in (dict(cached_lens=torch.zeros(3, dtype=torch.int32)), dict(new_lens=fake(4)), dict(first_pos=fake(2)), dict(block_table=fake(12)),
               dict(block_table=fake(4, 3)), dict(kv_lens=fake(2)), dict(cu_new=fake(3)), dict(pos=fake(9)), dict(counts=fake(3)),
               dict(slots=fake(10, dtype=torch.int64)), dict(free_pages=fake(9, dtype=torch.float32)), dict(cached_lens=fake(6)[::2])):
        with pytest.raises(AssertionError):
            B.tr_page_map(**dict(ok, **kw))
    sh = shape(4, 2, 64)
    bf = torch.bfloat16
    ok = dict(shape=sh, rotary=None, q=fake(5, 4, 64, dtype=bf), k=fake(5, 2, 64, dtype=bf), v=fake(5, 2, 64, dtype=bf), q_norm=None, k_norm=None, eps=1e-6,
              pos=fake(5), slots=fake(5), q_out=fake(5, 4, 64, dtype=bf), pages=None, stream=0)
    for kw in (dict(q=fake(5, 4, 64)), dict(k=fake(5, 3, 64, dtype=bf)), dict(v=fake(4, 2, 64, dtype=bf)), dict(q=fake(5, 64, 4, dtype=bf).transpose(1, 2)),
               dict(q=fake(5, 256, dtype=bf)), dict(q_out=fake(5, 8, 64, dtype=bf)[:, :4]), dict(q_norm=fake(32, dtype=bf)),
               dict(k_norm=fake(64, dtype=torch.float32)), dict(pos=fake(4)), dict(slots=fake(6)), dict(k=fake(5, 2, 128, dtype=bf)[..., ::2])):
        with pytest.raises(AssertionError):
            B.tr_paged_append(**dict(ok, **kw))
    pg = pages(n_kv_heads=2, head_dim=64, head_stride=64)
    ok = dict(shape=sh, q=fake(3, 4, 64, dtype=bf), pages=pg, block_table=fake(3, 7), kv_lens=fake(3), window=0, n_sink=0, out=fake(3, 4, 64, dtype=bf),
              workspace=None, stream=0)
    for kw in (dict(q=fake(3, 4, 64, dtype=torch.float32)), dict(q=fake(2, 4, 64, dtype=bf)), dict(out=fake(3, 4, 32, dtype=bf)), dict(block_table=fake(4, 7)),
               dict(kv_lens=fake(2)), dict(kv_lens=fake(3, dtype=torch.int64)), dict(q=fake(3, 8, 64, dtype=bf)[:, :4])):
        with pytest.raises(AssertionError):
            B.tr_paged_decode_attn(**dict(ok, **kw))
    with pytest.raises(TypeError):
        B.tr_paged_decode_attn(**dict(ok, pages=sh))
