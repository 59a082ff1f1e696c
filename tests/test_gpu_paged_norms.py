"""The head norm of the paged append over the whole range of its types: squares beyond fp32 and weights far from one."""
import numpy as np
import pytest
import torch

from tests import paged_reference as R
from tests.test_gpu_paged import B, DT, EPS, check_append, ints, randn  # noqa: F401  (B: the fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dt,d", [("bf16", 64), ("bf16", 128), ("f32", 64), ("f32", 128)])
@pytest.mark.parametrize("layout", [0, 1])
def test_heads_whose_squares_are_beyond_fp32(B, dt, d, layout):
    """Heads of up to the type's largest number next to ordinary ones: y = x / sqrt(mean(x^2) + eps) * weight is of ordinary size."""
    tokens = 12
    q, k, v = (randn(tokens, h, d, seed=h, dtype=torch.float32).clamp(-3, 3) for h in (6, 2, 2))
    for x in (q, k):
        x[1] *= 1e18
        x[2] *= 5e18
        x[3] *= 1e19
        x[4] *= 2e19
        x[5] *= 1e30
        x[6] *= 1e38
        x[7, 1] *= 1e25     # one head of several
        x[8, 0, d - 1] = 3e38
        x[9, 1] = torch.finfo(DT[dt]).max
    check_append(B, dt, 6, 2, d, tokens, d, layout, data=[x.to(DT[dt]) for x in (q, k, v)], seed=8)


@pytest.mark.parametrize("dt,d", [("bf16", 128), ("f32", 64)])
@pytest.mark.parametrize("eps", [1.2e-38, 1.0, 1e36, 3.4e38])
def test_eps_of_any_size_next_to_them(B, dt, d, eps):
    q = torch.cat([randn(1, 2, d, seed=1, dtype=torch.float32).clamp(-3, 3) * x for x in (1e17, 1e18, 3e18, 1e19, 3e19, 1e25, 1e38)]).to(DT[dt])
    w, out = torch.ones(d, dtype=DT[dt]), torch.empty_like(q).cuda()
    B.tr_paged_append(B.make_shape(2, 1, d, dt, 1e4), B.tr_rotary_init(0, 0, 1e4), q.cuda(), None, None, w.cuda(), None, eps, None, None, out, None)
    want, mag = R.heads(q, w, eps, torch.zeros(len(q)), [], 0)
    R.assert_within(out, want, R.heads_bound(want, mag, DT[dt]), "eps of %g" % eps)


def test_infinite_and_nan_heads_stay_by_themselves(B):
    d = 128
    gs = B.make_shape(4, 2, d, "bf16", 1e4)
    q = randn(3, 4, d, seed=1, dtype=torch.bfloat16)
    w = torch.ones(d, dtype=torch.bfloat16).cuda()
    clean, out = torch.empty_like(q).cuda(), torch.empty_like(q).cuda()
    rotary = B.tr_rotary_init(0, 0, 1e4)
    B.tr_paged_append(gs, rotary, q.cuda(), None, None, w, None, EPS, None, None, clean, None)
    q[1, 2, 77], q[2, 0, 5], q[2, 0, 6] = float("inf"), float("nan"), float("inf")
    B.tr_paged_append(gs, rotary, q.cuda(), None, None, w, None, EPS, None, None, out, None)
    assert torch.isnan(out[2, 0]).all() and torch.isnan(out[1, 2, 77])
    assert (out[1, 2, :77] == 0).all() and (out[1, 2, 78:] == 0).all()
    out[1, 2], out[2, 0] = clean[1, 2], clean[2, 0]
    assert torch.equal(out, clean)


@pytest.mark.parametrize("dt,d", [("bf16", 128), ("f32", 64)])
def test_weights_far_from_one(B, dt, d):
    """x / rms is of ordinary size, whatever the weight: a weight times 1 / rms need not be a number that fp32 has."""
    q = randn(6, 2, d, seed=1, dtype=torch.float32)
    scale = torch.tensor([1e17, 1.0, 1e-3, 1e-10, 0.0, 1e10])
    q = (q * scale[:, None, None]).to(DT[dt])
    gs = B.make_shape(2, 1, d, dt, 1e4)
    for size in (1e-30, 1e30, 2e36):
        w = (randn(d, seed=3, dtype=torch.float32).clamp(-2, 2) * size).to(DT[dt])
        out = torch.empty_like(q).cuda()
        B.tr_paged_append(gs, B.tr_rotary_init(0, 0, 1e4), q.cuda(), None, None, w.cuda(), None, EPS, None, None, out, None)
        want, mag = R.heads(q, w, EPS, torch.zeros(6), [], 0)
        R.assert_within(out, want, R.heads_bound(want, mag, DT[dt]), "weight of %g" % size)
