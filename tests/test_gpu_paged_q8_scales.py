"""The calls over a paged cache in 8 bits with scales at the ends of their range, those that an append writes (bytes 10 to 247) and the others that are
read for what they mean."""
import numpy as np
import pytest
import torch

from tests import paged_q8_reference as Q
from tests import paged_reference as R
from tests.test_gpu_paged import DT, ints, randn, tables
from tests.test_gpu_paged_q8 import EPS, run_read
from tests.test_gpu_paged_q8_decode import run

pytestmark = pytest.mark.gpu
BYTES = np.arange(1, 255)
LEAST_NORMAL = 2.0 ** -126


@pytest.fixture(scope="module")
def B():
    from paper_2410_07590_amd import binding
    binding.lib()
    return binding


def codes_of_every_scale(hk, d, seed):
    """A page of 16 rows for each byte from 1 to 254, with codes whose values are zero or normal numbers at it."""
    rng = np.random.default_rng(seed)
    codes = np.zeros((len(BYTES), 16, hk, d), np.uint8)
    for i, s in enumerate(BYTES):
        worth = Q.VALUES.numpy() * 2.0 ** (int(s) - 127)
        codes[i] = rng.choice(np.flatnonzero((worth == 0) | ((abs(worth) >= LEAST_NORMAL) & (abs(worth) < 2.0 ** 128))), codes.shape[1:])
    scale = np.repeat(BYTES.astype(np.uint8), hk).reshape(-1, hk, 1)
    return torch.from_numpy(codes), torch.from_numpy(scale)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
def test_read_back_at_every_scale(B, dt, d):
    hk, n = 2, len(BYTES)
    (k, ks), (v, vs) = (codes_of_every_scale(hk, d, i) for i in (1, 2))
    got = run_read(B, dt, hk, d, k.cuda(), v.cuda(), ks.cuda(), vs.cuda(), np.arange(n)[:, None], [16] * n, 16 * np.arange(n + 1), 16 * n)
    for out, codes, scale in ((got[0], k, ks), (got[1], v, vs)):
        assert torch.equal(out, Q.values(codes, scale).reshape(16 * n, hk, d))


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("hq,hk,d", [(4, 2, 64), (6, 2, 128), (34, 1, 64), (20, 1, 128)])
def test_the_only_key_of_any_scale_gives_its_value(B, dt, hq, hk, d):
    """Bit for bit: the weight is 1, its other parts are 0, and so are the weights of all other keys of the unit."""
    n = len(BYTES)
    (k, ks), (v, vs) = (codes_of_every_scale(hk, d, i) for i in (1, 2))
    q = randn(n, hq, d, seed=5, dtype=torch.float32) * torch.where(torch.arange(n) < n // 2, 1.0, 2.0 ** -60)[:, None, None]   # finite scores
    got = run(B, B.make_shape(hq, hk, d, dt, 1e4), q.to(DT[dt]).cuda(), k.cuda(), v.cuda(), ks.cuda(), vs.cuda(), ints(np.arange(n)[:, None]), ints([1] * n))
    want = Q.values(v, vs)[:, 0].repeat_interleave(hq // hk, 1)
    assert torch.equal(got.cpu().double(), want)


LENS = [1, 12, 3, 200, 65]


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("top", [13, 40, 90, 127, 200, 230, 237, 242, 246, 247])
def test_keys_of_any_scale_against_queries_of_the_inverse(B, dt, d, top):
    """Scores of size 1 from keys whose largest scale is the byte `top` and queries that are as small or as large as that needs, subnormal ones
    among them."""
    hq, hk, page = 8, 2, 16
    table, n_pages = tables(np.random.default_rng(top), LENS, page)
    (k, ks), (v, vs) = (Q.random_pool(n_pages, page, hk, d, i, 1) for i in (1, 2))
    shift = top - int(ks.max())
    ks = (ks.int() + shift).to(torch.uint8)
    assert int(ks.min()) >= 10
    if top == 247:   # what is larger at this scale is beyond fp32, and an append never leaves it
        k = (k & 128) | (k & 127).clamp(max=0x77)
    q = torch.ldexp(torch.randn(len(LENS), hq, d, generator=torch.Generator().manual_seed(top), dtype=torch.float64), torch.tensor(-shift)).to(DT[dt])
    got = run(B, B.make_shape(hq, hk, d, dt, 1e4), q.cuda(), k.cuda(), v.cuda(), ks.cuda(), vs.cuda(), ints(table), ints(LENS))
    # what the queries are, at a size where nothing is lost
    want, bound = R.decode_batch(torch.ldexp(q.double(), torch.tensor(shift)), Q.values(k, (ks.int() - shift).to(torch.uint8)), Q.values(v, vs), torch.from_numpy(table), LENS,
                                 0, 0, hq // hk)
    R.assert_within(got, want, torch.finfo(DT[dt]).eps / 2 * want.abs() * 1.01 + bound, "attention")


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("top", [10, 12, 30, 127, 238, 247, 251, 254])
def test_values_of_any_scale(B, dt, d, top):
    """Sums stay below the largest fp32 number: at most 12 keys of up to 448 * 2^(238 - 127) < 2^120, and of blocks with larger scales codes that
    are less.  What is below the least normal number may be taken as zero: three products of a key's weight with its value and their sums, and the result."""
    hq, hk, page, lens = 8, 2, 16, [1, 12, 3, 7, 2]
    table, n_pages = tables(np.random.default_rng(top), lens, page)
    (k, ks), (v, vs) = (Q.random_pool(n_pages, page, hk, d, i, 0) for i in (1, 2))
    shift = top - int(vs.max())
    vs = (vs.int() + shift).clamp(1, 254).to(torch.uint8)
    if top > 238:
        v = Q.round_code(torch.ldexp(Q.VALUES[v.long()], torch.tensor(238 - top)))
    worth = Q.values(v, vs)
    v = torch.where((worth == 0) | (worth.abs() >= LEAST_NORMAL), v, 0)
    worth = Q.values(v, vs)
    assert float(worth.abs().max()) * 12 < 2.0 ** 128
    q = randn(len(lens), hq, d, seed=5, dtype=DT[dt])
    got = run(B, B.make_shape(hq, hk, d, dt, 1e4), q.cuda(), k.cuda(), v.cuda(), ks.cuda(), vs.cuda(), ints(table), ints(lens))
    # in units that keep the sums of the definition in the range of 64 bits without any loss
    want, bound = R.decode_batch(q, Q.values(k, ks), worth, torch.from_numpy(table), lens, 0, 0, hq // hk)
    R.assert_within(got, want, torch.finfo(DT[dt]).eps / 2 * want.abs() * 1.01 + bound + (6 * 12 + 1) * LEAST_NORMAL, "attention")


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("first", [1, 9])
def test_append_to_blocks_of_any_scale(B, dt, first):
    """A row of ordinary, of the smallest and of the largest values for blocks whose scales are every byte from 1 to 254: the scale grows to what the
    row needs and to the least that an append writes, or stays."""
    hk, d, n = 3, 64, len(BYTES)
    (k0, ks0), (v0, vs0) = (codes_of_every_scale(hk, d, i) for i in (1, 2))
    k = randn(n, hk, d, seed=first, dtype=torch.float32)
    k[:, 1] *= 2.0 ** -120
    k[:, 2] = k[:, 2].sign() * torch.finfo(torch.float32).max * torch.linspace(0.5, 1, d)
    k = k.clamp(-torch.finfo(DT[dt]).max, torch.finfo(DT[dt]).max).to(DT[dt])
    v = k.flip(1).contiguous()
    slots = 16 * np.arange(n) + first
    gk, gv, gks, gvs = k0.cuda(), v0.cuda(), ks0.cuda(), vs0.cuda()
    B.tr_paged_append_q8(B.make_shape(hk, hk, d, dt, 1e4), B.tr_rotary_init(1, 0, 1e4), None, k.cuda(), v.cuda(), None, None, EPS, None, ints(slots), None,
                         B.make_pages_q8(gk, gv, gks, gvs))
    torch.cuda.synchronize()
    Q.check_append(gk.cpu(), gks.cpu(), k0, ks0, k.double(), 0, slots, "keys")
    Q.check_append(gv.cpu(), gvs.cpu(), v0, vs0, v.double(), 0, slots, "values")
