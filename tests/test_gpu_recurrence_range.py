"""Recurrences at and behind the ends of binary32: infinite states and gradients, factors whose products pass the range while the states do not, factors above
1; in every form of the launch (one tile; tiles one after the other, with one channel and with two in a lane; tiles in workgroups of their own)."""
import pytest
import torch

from recurrent_util import recurrence_grad64
from test_gpu_linear_recurrence import MODES, case, check, check_grad
from train_util import DEV, assert_within, half_ulp, rand, smallest

pytestmark = pytest.mark.gpu

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
# steps, batch, channels; steps are multiples of 18
FORMS = [(18, 3, 70, F32), (126, 3, 70, F16), (306, 3, 70, F32), (306, 3, 70, BF16), (306, 1, 17001, F32), (306, 3, 11002, BF16), (3006, 3, 70, F32),
         (3006, 3, 70, F16), (20016, 1, 33, BF16)]


@pytest.fixture(scope="module")
def amq():
    import paper_1802_00150_amd as amq
    return amq


def forward(amq, gate, x, h0, mode, lengths=None):
    hs, last, states = amq.linear_recurrence(gate.to(DEV), x.to(DEV), h0.to(DEV), mode=mode, lengths=None if lengths is None else lengths.to(DEV), states=True)
    return hs.cpu(), last.cpu(), None if states is None else states.cpu()


def backward(amq, dhs, gate, x, h0, states, dl, mode, lengths=None):
    out = amq.linear_recurrence_backward(dhs.to(DEV), gate.to(DEV), x.to(DEV), h0.to(DEV), None if states is None else states.to(DEV), dl.to(DEV), mode=mode,
                                         lengths=None if lengths is None else lengths.to(DEV))
    return [t.cpu() for t in out]


def same_but(got, want, channels):
    """Bit for bit, NaN like NaN, but for these channels."""
    keep = torch.ones(got.shape[-1], dtype=torch.bool)
    keep[channels] = False
    return torch.equal(torch.nan_to_num(got[..., keep], 7.0), torch.nan_to_num(want[..., keep], 7.0))


def ragged(T, B):
    return torch.tensor([T, max(1, T // 2 + 3), max(1, T - 9)][:B])


@pytest.mark.parametrize("T,B,n,dtype", FORMS)
@pytest.mark.parametrize("mode", MODES)
@pytest.mark.parametrize("padded", [False, True])
def test_infinite_states(amq, T, B, n, dtype, mode, padded):
    """An infinity stays one, whatever the gates' signs, until another of the other sign meets it."""
    gate, x, h0 = case(T + n, T, B, n, dtype, mode)
    if mode == "decay":
        gate = gate.abs()
    lengths = ragged(T, B) if padded else None
    good = forward(amq, gate, x, h0, mode, lengths)
    bad_h, bad_x = h0.clone(), x.clone()
    bad_h[:, 3], bad_h[:, 32] = float("inf"), -float("inf")
    first, second = T // 3, T // 2
    bad_x[first, :, 5] = float("inf")
    bad_x[second, :, 5] = -float("inf")
    hs, last, states = forward(amq, gate, bad_x, bad_h, mode, lengths)
    channels = [3, 5, 32]
    assert same_but(hs, good[0], channels) and same_but(last, good[1], channels)
    for b in range(B):
        end = T if lengths is None else int(lengths[b])
        assert bool((hs[:end, b, 3] == float("inf")).all()) and bool((hs[:end, b, 32] == -float("inf")).all())
        assert torch.equal(hs[:first, b, 5], good[0][:first, b, 5])
        assert bool((hs[first:second, b, 5] == float("inf")).all()) and bool(torch.isnan(hs[second:end, b, 5]).all())
        assert bool((hs[end:, b] == 0).all())
        # (the shortest entry of 18 steps ends in front of the second)
        assert bool(torch.isnan(last[b, 5])) if end > second else float(last[b, 5]) == float("inf")
    assert bool((last[:, 3] == float("inf")).all()) and bool((last[:, 32] == -float("inf")).all())
    if states is not None and lengths is None:
        assert same_but(states, good[2], channels) and bool((states[:, :, 3] == float("inf")).all())


@pytest.mark.parametrize("T,B,n,dtype", FORMS)
@pytest.mark.parametrize("mode", MODES)
@pytest.mark.parametrize("padded", [False, True])
def test_infinite_gradients(amq, T, B, n, dtype, mode, padded):
    """An infinite gradient of the last state is one of every step; an infinite state makes the gates' gradients infinite and leaves the others as they are."""
    gate, x, h0 = case(T + n, T, B, n, dtype, mode)
    if mode == "decay":
        gate = gate.abs()
    lengths = ragged(T, B) if padded else None
    dhs, dl = rand(1, T, B, n).to(dtype), rand(2, B, n)
    states = forward(amq, gate, x, h0, mode, lengths)[2]
    good = backward(amq, dhs, gate, x, h0, states, dl, mode, lengths)
    behind = torch.zeros(T, B, dtype=torch.bool) if lengths is None else torch.arange(T)[:, None] >= lengths
    bad = dl.clone()
    bad[:, 4] = float("inf")
    dg, dx, dh0 = backward(amq, dhs, gate, x, h0, states, bad, mode, lengths)
    assert same_but(dg, good[0], [4]) and same_but(dx, good[1], [4]) and same_but(dh0, good[2], [4])
    assert bool((dx[..., 4].masked_fill(behind, float("inf")) == float("inf")).all()) and bool((dh0[:, 4] == float("inf")).all())
    assert bool((dg[..., 4].abs().masked_fill(behind, float("inf")) == float("inf")).all())
    assert bool((dx[..., 4][behind] == 0).all()) and bool((dg[..., 4][behind] == 0).all())
    bad = h0.clone()
    bad[:, 5] = float("inf")
    states = forward(amq, gate, x, bad, mode, lengths)[2]
    dg, dx, dh0 = backward(amq, dhs, gate, x, bad, states, dl, mode, lengths)
    assert same_but(dg, good[0], [5]) and same_but(dx, good[1], [5]) and same_but(dh0, good[2], [5])
    assert bool((dg[..., 5].abs().masked_fill(behind, float("inf")) == float("inf")).all()) and bool((dg[..., 5][behind] == 0).all())
    part = [t[..., 5:6].double().masked_fill(behind[..., None], 0.0) for t in (dhs, gate, x)]
    ref, tol = recurrence_grad64(*part, h0[:, 5:6].double(), dl[:, 5:6].double(), mode, lengths)
    assert_within(dx[..., 5:6], ref[1], tol[1] + half_ulp(dtype) * ref[1].abs() + smallest(dtype), "dx")
    assert_within(dh0[:, 5:6], ref[2], tol[2], "dh0")


@pytest.mark.parametrize("T,B,n,dtype", FORMS)
def test_products_of_factors_beyond_the_range(amq, T, B, n, dtype):
    """Nine factors of 2^15 and nine of 2^-15 in turn: a state goes from 2^-125 to 2^10 and back, and its gradient from 2^10 to 2^-125, while the
    factors' product passes 2^128.  All of them are powers of two, so the results are exact (below 2^-126 they may be 0).  A state of 0 stays 0."""
    gate, x, h0 = case(T + n, T, B, n, dtype, "decay")
    up = torch.tensor([2.0 ** 15] * 9 + [2.0 ** -15] * 9).repeat(T // 18)
    dhs, dl = rand(1, T, B, n).to(dtype), rand(2, B, n)
    for t in (gate, x, dhs, h0, dl):
        t[..., 7] = t[..., 32] = 0
    good = forward(amq, gate, x, h0, "decay")
    good_grads = backward(amq, dhs, gate, x, h0, good[2], dl, "decay")
    gate[..., 7] = gate[..., 32] = up[:, None].to(dtype)
    h0[:, 7], dl[:, 7] = 2.0 ** -125, 2.0 ** 10
    hs, last, states = forward(amq, gate, x, h0, "decay")
    exact = (2.0 ** -125 * torch.cumprod(up.double(), 0))[:, None].expand(T, B)
    channels = [7, 32]
    assert same_but(hs, good[0], channels) and same_but(last, good[1], channels)
    assert_within(hs[..., 7], exact.to(dtype).double(), torch.where(exact < 2.0 ** -125, 2.0 ** -126, 0.0), "hs")
    assert bool((last[:, 7] == 2.0 ** -125).all()) and bool((hs[..., 32] == 0).all()) and bool((last[:, 32] == 0).all())
    if states is not None:
        assert torch.equal(states[:, :, 7].double(), exact[127:T - 1:128]) and bool((states[:, :, 32] == 0).all())
    dg, dx, dh0 = backward(amq, dhs, gate, x, h0, states, dl, "decay")
    assert same_but(dg, good_grads[0], channels) and same_but(dx, good_grads[1], channels) and same_but(dh0, good_grads[2], channels)
    e = torch.cat([torch.cumprod(up.double().flip(0), 0).flip(0)[1:], torch.ones(1, dtype=torch.float64)]) * 2.0 ** 10
    assert_within(dx[..., 7], e[:, None].expand(T, B).to(dtype).double(), torch.where(e < 2.0 ** -125, 2.0 ** -126, 0.0)[:, None].expand(T, B), "dx")
    before = torch.cat([torch.full((1, B), 2.0 ** -125, dtype=torch.float64), exact[:-1]])
    assert_within(dg[..., 7], (e[:, None] * before).to(dtype).double(), torch.full((T, B), 2.0 ** -126, dtype=torch.float64), "dgate")
    assert bool((dh0[:, 7] == 2.0 ** 10).all())
    assert bool((dx[..., 32] == 0).all()) and bool((dg[..., 32] == 0).all()) and bool((dh0[:, 32] == 0).all())


@pytest.mark.parametrize("T,B,n,dtype", FORMS)
def test_factors_above_one(amq, T, B, n, dtype):
    """States that grow by 1.05 a step for 150 steps and shrink by 0.95 for 200, of either sign, against binary64."""
    _, x, h0 = case(T, T, B, n, dtype, "decay")
    x = (x.float() / 64).to(dtype)
    grows = (torch.arange(T)[:, None, None] + torch.arange(n)) % 350 < 150
    sign = torch.where(rand(3, n) > -0.5, 1.0, -1.0)
    gate = (torch.where(grows, 1.05, 0.95) * sign).expand(T, B, n).to(dtype).contiguous()
    check(amq, gate, x, h0, "decay")
    check_grad(amq, gate, x, h0, "decay")


def test_states_next_to_the_range(amq):
    """h and x of 3e38: f h + (1 - f) x stays below the larger of the two although h + (1 - f) x does not."""
    for T, n in ((5, 64), (300, 64), (3000, 64)):
        gate, x = torch.linspace(-4, 4, n).expand(T, 1, n).contiguous(), torch.full((T, 1, n), 3e38)
        hs, last, _ = forward(amq, gate, x, torch.full((1, n), 3e38), "blend")
        ref, tol = 3e38, 3e38 * 2.0 ** -24
        # (each step is off by the roundings of f, 1 - f and of the sum: less than 24 of them; an error decays by f)
        f = torch.sigmoid(gate.double())
        assert_within(hs, torch.full_like(f, ref), 24 * tol / (1 - f), "hs")


def test_neither_form_of_the_launch_decides(amq):
    """A channel's overflow does not depend on how many others there are."""
    T = 1000
    gate = torch.full((T, 1, 1), 2.0)
    gate[500:] = 0.5
    x = torch.zeros(T, 1, 1)
    x[600] = 1.0
    want = torch.cat([torch.zeros(600), 0.5 ** torch.arange(400.0)])
    for B, n in ((1, 1), (3, 70), (1, 20000)):
        hs, last, states = forward(amq, gate.expand(T, B, n).contiguous(), x.expand(T, B, n).contiguous(), torch.zeros(B, n), "decay")
        assert_within(hs, want.double()[:, None, None].expand(T, B, n), torch.full((T, B, n), 2.0 ** -126, dtype=torch.float64), "hs")
