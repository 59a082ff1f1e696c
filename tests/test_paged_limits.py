"""The limits that the header states for tr_paged_decode_attn, at both sides of each, no GPU needed: sizes within them have a workspace,
sizes beyond are refused with the code that stands beside the limit."""
import ctypes as C

import pytest

from paper_2410_07590_amd import binding as B

AT = [0x7000_0000_0000 + (i << 44) for i in range(7)]   # 16 TiB apart


def status(dtype, hq, hk, d, n_req, blocks, page):
    """Without a workspace: what is within the limits needs one."""
    sh = B.tr_shape(hq, hk, d, dtype, 1e4, 0, 0)
    pg = B.tr_pages(AT[0], AT[1], 0, d, page * d, 1, page, hk, d, dtype, 0)
    i, p = C.c_int32, C.c_void_p
    return B.lib().tr_paged_decode_attn(C.byref(sh), p(AT[2]), C.byref(pg), p(AT[3]), i(blocks), p(AT[4]), i(n_req), i(0), i(0), p(AT[5]), None,
                                        C.c_size_t(0), None)


@pytest.mark.parametrize("dtype,hq,hk,d,n_req,blocks,page,beyond", [
    (B.TR_BF16, 4, 4, 64, 1, 2 ** 20, 1024, B.TR_ERR_INVALID_ARG),          # 2^30 keys
    (B.TR_F32, 4, 4, 64, 1, 2 ** 27, 8, B.TR_ERR_INVALID_ARG),
    (B.TR_BF16, 28, 4, 128, 256, 2 ** 15, 1024, B.TR_ERR_UNSUPPORTED),      # 1024 items of 2^20 units
    (B.TR_BF16, 128, 4, 128, 256, 2 ** 15, 1024, B.TR_ERR_UNSUPPORTED),     # 32 query heads to a KV head are still one block
    (B.TR_BF16, 132, 4, 128, 128, 2 ** 15, 1024, B.TR_ERR_UNSUPPORTED),     # 33 are two
    (B.TR_F32, 28, 4, 128, 256, 2 ** 15, 512, B.TR_ERR_UNSUPPORTED)])       # units of 16
def test_keys_that_a_table_has_room_for(dtype, hq, hk, d, n_req, blocks, page, beyond):
    for at, want in ((blocks, B.TR_ERR_WORKSPACE), (blocks + 1, beyond)):
        assert status(dtype, hq, hk, d, n_req, at, page) == want
        size = B.tr_paged_decode_attn_workspace_size(B.tr_shape(hq, hk, d, dtype, 1e4, 0, 0), n_req, at, page)
        assert (size > 0) == (at == blocks)


@pytest.mark.parametrize("heads,n_req,beyond_heads,beyond_n", [(1, 65536, 1, 65537), (255, 65536, 256, 65536), (2 ** 24 - 1, 1, 2 ** 24, 1)])
def test_requests_and_heads(heads, n_req, beyond_heads, beyond_n):
    assert status(B.TR_BF16, heads, heads, 64, n_req, 8, 16) == B.TR_ERR_WORKSPACE
    assert status(B.TR_BF16, beyond_heads, beyond_heads, 64, beyond_n, 8, 16) == B.TR_ERR_UNSUPPORTED
