"""Clipping to limits that binary32 does not hold."""
import math

import pytest
import torch

from train_util import DEV, U, assert_within, rand

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def amq():
    import paper_1802_00150_amd as amq
    return amq


def test_the_limit_is_not_rounded(amq):
    """Two roundings: the factor's and the product's.  (A limit rounded to binary32 makes three of them, over 2 U in some of these cases.)"""
    three = 0
    for k in range(200):
        g = rand(k, 64)
        limit = 0.3 + 1e-3 * k + 2.0 ** -27
        norm = math.sqrt(float(g.double().square().sum()))
        ref = g.double() * (limit / norm)
        out = torch.empty(64, device=DEV)
        amq.clip_gradients([g.to(DEV)], limit, out=[out])
        assert_within(out, ref, 2 * U * (1 + U) * ref.abs(), "limit %d" % k)
        rounded = g * torch.tensor(float(torch.tensor(limit)) / norm)
        three += bool(((rounded.double() - ref).abs() > 2 * U * (1 + U) * ref.abs()).any())
    assert three


def test_limits_beyond_the_range(amq):
    """Limits that binary32 would hold as infinity or 0."""
    g = torch.tensor([3e38, -1e38, 2e38] * 100, device=DEV)
    norm = math.sqrt(float(g.cpu().double().square().sum()))
    out = torch.empty_like(g)
    for limit in (1e39, norm * 2, 1e300):
        amq.clip_gradients([g], limit, out=[out])
        ref = g.cpu().double() * min(1.0, limit / norm)
        assert_within(out, ref, 2 * U * (1 + U) * ref.abs(), "limit %g" % limit)
    tiny = torch.tensor([1e30, -3e30], device=DEV)
    out = torch.empty_like(tiny)
    amq.clip_gradients([tiny], 1e-50, out=[out])
    assert bool((out == 0).all())
    big = torch.full((2,), 2.0 ** 100, device=DEV)
    amq.clip_gradients([big], 1e-46, out=[out[:2]])
    assert bool((out == 0).all())
    with pytest.raises(amq.AmqError):
        amq.clip_gradients([tiny], -1e-60)
