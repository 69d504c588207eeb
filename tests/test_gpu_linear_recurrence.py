"""Linear recurrences, forward and backward, against the formulas in binary64 (tolerances: recurrent_util)."""
import pytest
import torch

from recurrent_util import recurrence64, recurrence_grad64
from train_util import DEV, DTYPES, U, assert_within, half_ulp, rand, smallest

pytestmark = pytest.mark.gpu

MODES = ["blend", "decay"]
# steps, batch, channels: one of each, part of a wave's 8 steps, a tile's 128, the states' positions, many tiles; pieces that end inside a row
SIZES = [(1, 1, 1), (1, 3, 5), (1, 2, 1024), (7, 2, 64), (8, 1, 65), (9, 2, 127), (35, 4, 33), (64, 1, 300), (127, 1, 130), (128, 2, 64), (129, 2, 66),
         (130, 1, 1), (257, 1, 3), (700, 2, 70), (1000, 3, 129), (2500, 1, 40), (9000, 1, 2)]


@pytest.fixture(scope="module")
def amq():
    import paper_1802_00150_amd as amq
    return amq


def case(seed, T, B, n, dtype, mode):
    gate, x = rand(seed, T, B, n) * 1.5 + torch.linspace(-3, 6, n), rand(seed + 1, T, B, n)
    if mode == "decay":
        gate = torch.sigmoid(gate) * torch.where(rand(seed + 2, n) > -0.5, 1.0, -1.0)
        x = x * (1 - gate.abs())
    return gate.to(dtype), x.to(dtype), rand(seed + 3, B, n)


def padded(T, B):
    """Lengths with none, one, all and something between; out of range ones count as none and all."""
    some = [0, T, max(1, T // 3), 1, -5, T + 7, max(0, T - 1), T // 2]
    return torch.tensor([some[b % len(some)] for b in range(B)])


def check(amq, gate, x, h0, mode, lengths=None, views=None, what=""):
    dtype = x.dtype
    T, B, n = x.shape
    on = lambda t: None if t is None else t.to(DEV)  # noqa: E731
    g, v = views if views else (gate.to(DEV), x.to(DEV))
    hs, last, states = amq.linear_recurrence(g, v, on(h0), mode=mode, lengths=on(lengths), states=True)
    clean = [t.double() for t in (gate, x)]
    if lengths is not None:
        clean = [t.masked_fill((torch.arange(T)[:, None] >= lengths)[:, :, None], 0.0) for t in clean]
    h = torch.zeros(B, n, dtype=torch.float64) if h0 is None else h0.double()
    ref, tol, _ = recurrence64(clean[0], clean[1], h, mode, lengths)
    behind = torch.zeros(T, B, 1, dtype=torch.bool) if lengths is None else (torch.arange(T)[:, None] >= lengths)[:, :, None]
    out = ref.masked_fill(behind, 0.0)
    assert_within(hs, out, (tol + half_ulp(dtype) * ref.abs() + smallest(dtype)).masked_fill(behind, 0.0), what + " hs")
    assert hs.dtype == dtype and last.dtype == torch.float32
    assert_within(last, ref[-1], tol[-1], what + " h_last")
    if T > 128:
        at = torch.arange(127, T - 1, 128)
        # (those behind an entry's end are not written)
        unused = torch.zeros(len(at), B, n, dtype=torch.bool) if lengths is None else (at[:, None] + 1 >= lengths)[:, :, None].expand(-1, -1, n)
        assert_within(states.cpu().masked_fill(unused, 0.0), ref[at].masked_fill(unused, 0.0), tol[at], what + " states")
    else:
        assert states is None
    return hs, last, states


def check_grad(amq, gate, x, h0, mode, lengths=None, dh_last=True, seed=0, states=None, outs=(None, None), views=None, what=""):
    dtype = x.dtype
    T, B, n = x.shape
    on = lambda t: None if t is None else t.to(DEV)  # noqa: E731
    dhs, dl = rand(seed + 7, T, B, n).to(dtype), rand(seed + 8, B, n) if dh_last else None
    behind = torch.zeros(T, B, 1, dtype=torch.bool) if lengths is None else (torch.arange(T)[:, None] >= lengths)[:, :, None]
    g, v = views if views else (gate.to(DEV), x.to(DEV))
    if states is None:
        states = amq.linear_recurrence(g, v, on(h0), mode=mode, lengths=on(lengths), states=True)[2]
    dg, dx, dh0 = amq.linear_recurrence_backward(dhs.masked_fill(behind, float("nan")).to(DEV), g, v, on(h0), states, on(dl), mode=mode, lengths=on(lengths),
                                                 dgate=outs[0], dx=outs[1])
    zero = torch.zeros(B, n, dtype=torch.float64)
    args = [t.double().masked_fill(behind, 0.0) for t in (dhs, gate, x)]
    ref, tol = recurrence_grad64(*args, zero if h0 is None else h0.double(), zero if dl is None else dl.double(), mode, lengths)
    for name, got, r, t in (("dgate", dg, ref[0], tol[0]), ("dx", dx, ref[1], tol[1])):
        assert got.dtype == dtype
        assert_within(got, r, (t + half_ulp(dtype) * r.abs() + smallest(dtype)).masked_fill(behind, 0.0), what + " " + name)
    if h0 is None:
        assert dh0 is None
    else:
        assert_within(dh0, ref[2], tol[2], what + " dh0")


@pytest.mark.parametrize("T,B,n", SIZES)
@pytest.mark.parametrize("mode", MODES)
@pytest.mark.parametrize("dtype", DTYPES)
def test_sizes(amq, T, B, n, mode, dtype):
    gate, x, h0 = case(T + n, T, B, n, dtype, mode)
    what = "%dx%dx%d" % (T, B, n)
    check(amq, gate, x, h0, mode, what=what)
    check_grad(amq, gate, x, h0, mode, what=what)


@pytest.mark.parametrize("T,B,n", [(1, 8, 3), (7, 8, 64), (35, 8, 130), (128, 8, 2), (129, 8, 65), (400, 9, 100), (1500, 8, 33), (300, 260, 70), (140, 300, 128)])
@pytest.mark.parametrize("mode", MODES)
@pytest.mark.parametrize("dtype", DTYPES)
def test_lengths(amq, T, B, n, mode, dtype):
    """Padding holds NaN and infinities, which reach nothing."""
    gate, x, h0 = case(T + n, T, B, n, dtype, mode)
    lengths = padded(T, B)
    behind = (torch.arange(T)[:, None] >= lengths)[:, :, None]
    gate, x = gate.masked_fill(behind, float("nan")), x.masked_fill(behind, float("inf"))
    check(amq, gate, x, h0, mode, lengths)
    check_grad(amq, gate, x, h0, mode, lengths)


@pytest.mark.parametrize("mode", MODES)
@pytest.mark.parametrize("dtype", DTYPES)
def test_without_first_state_and_last_gradient(amq, mode, dtype):
    for T in (3, 200):
        gate, x, _ = case(T, T, 2, 50, dtype, mode)
        check(amq, gate, x, None, mode)
        check_grad(amq, gate, x, None, mode, dh_last=False)


@pytest.mark.parametrize("mode", MODES)
def test_channels_enough_for_the_card(amq, mode):
    """Tiles one after the other in one workgroup, with one channel and with two in a lane."""
    for T, B, n, dtype in ((137, 1, 40001, torch.bfloat16), (260, 3, 22100, torch.bfloat16), (400, 1, 17001, torch.float32), (300, 1, 8192, torch.float16)):
        gate, x, h0 = case(T, T, B, n, dtype, mode)
        check(amq, gate, x, h0, mode)
        check_grad(amq, gate, x, h0, mode)


def layouts(gate, x):
    """The same tensors as columns of one projection, batch first, and as a slice of more steps, entries and channels at an odd offset."""
    T, B, n = x.shape
    wide = torch.cat([gate, x], 2).to(DEV)
    yield "columns", (wide[:, :, :n], wide[:, :, n:])
    first = [t.transpose(0, 1).contiguous().to(DEV).transpose(0, 1) for t in (gate, x)]
    yield "batch first", first
    large = torch.full((2, T + 2, B + 3, n + 5), float("nan"), dtype=x.dtype, device=DEV)
    inner = [large[i, 1:T + 1, 2:B + 2, 3:n + 3] for i in (0, 1)]
    inner[0].copy_(gate)
    inner[1].copy_(x)
    yield "slice", inner


@pytest.mark.parametrize("T,B,n", [(1, 3, 7), (5, 1, 64), (35, 4, 131), (300, 3, 66), (140, 300, 66)])
@pytest.mark.parametrize("mode", MODES)
@pytest.mark.parametrize("dtype", DTYPES)
def test_layouts(amq, T, B, n, mode, dtype):
    gate, x, h0 = case(T + n, T, B, n, dtype, mode)
    for name, views in layouts(gate, x):
        hs, last, _ = check(amq, gate, x, h0, mode, views=views, what=name)
        # results beside each other in one buffer whose other entries stay as they are
        room = torch.full((B, T, 3 * n + 1), 7.0, dtype=dtype, device=DEV)
        a, b, c = (room[:, :, i * n + 1:(i + 1) * n + 1].transpose(0, 1) for i in range(3))
        out, _, _ = amq.linear_recurrence(*views, h0.to(DEV), mode=mode, out=a)
        assert out is a and torch.equal(a, hs)
        check_grad(amq, gate, x, h0, mode, views=views, outs=(b, c), what=name)
        assert torch.equal(a, hs) and bool((room[:, :, 0] == 7.0).all())


@pytest.mark.parametrize("mode", MODES)
def test_broadcast_operands(amq, mode):
    """A gate that all entries share, a candidate that all steps share."""
    gate, x, h0 = case(1, 40, 3, 70, torch.float32, mode)
    g, v = gate[:, :1].expand(40, 3, 70), x[:1].expand(40, 3, 70)
    views = gate[:, :1].to(DEV).expand(40, 3, 70), x[:1].to(DEV).expand(40, 3, 70)
    check(amq, g, v, h0, mode, views=views)
    check_grad(amq, g, v, h0, mode, views=views)


@pytest.mark.parametrize("mode", MODES)
@pytest.mark.parametrize("dtype", DTYPES)
def test_state_in_place_and_sequences_in_parts(amq, mode, dtype):
    """A sequence in parts with its state handed on in place, down to single tokens, is the sequence in one call but for the folds' roundings."""
    T, B, n = 150, 3, 67
    gate, x, h0 = case(5, T, B, n, dtype, mode)
    whole, tol, _ = recurrence64(gate.double(), x.double(), h0.double(), mode)
    g, v = gate.to(DEV), x.to(DEV)
    for parts in ([1] * 20 + [130], [149, 1], [7, 128, 15]):
        h, at, got = h0.to(DEV), 0, []
        for part in parts:
            hs, last, _ = amq.linear_recurrence(g[at:at + part], v[at:at + part], h, mode=mode, h_out=h)
            assert last is h
            got.append(hs)
            at += part
        assert_within(torch.cat(got), whole, tol + half_ulp(dtype) * whole.abs() + smallest(dtype), str(parts))
        assert_within(h, whole[-1], tol[-1], "state")


def test_extreme_gates(amq):
    """Gates at and far behind the ends of the exponential's range: f is 0 or 1, the state is x or stays."""
    gate = torch.tensor([[float("inf"), 200.0, 100.0, 88.0, -88.0, -100.0, -200.0, -float("inf")]]).repeat(40, 1)[:, None]
    x, h0 = torch.full((40, 1, 8), 1e-3), torch.full((1, 8), 1e6)
    hs, last, _ = amq.linear_recurrence(gate.to(DEV), x.to(DEV), h0.to(DEV))
    assert torch.equal(last.cpu()[0, :4], h0[0, :4]) and torch.equal(last.cpu()[0, 4:], x[0, 0, 4:])
    assert torch.equal(hs.cpu()[:, 0, :4], h0[:, :4].expand(40, 4)) and bool((hs.cpu()[1:, 0, 4:] == 1e-3).all())
    dg, dx, dh0 = amq.linear_recurrence_backward(torch.ones(40, 1, 8, device=DEV), gate.to(DEV), x.to(DEV), h0.to(DEV))
    assert bool(torch.isfinite(dg).all()) and bool((dx[..., :2] == 0).all()) and bool((dx[..., 6:] == 1).all())
    assert bool((dh0[:, :2] == 40).all()) and bool((dh0[:, 6:] == 0).all())


def test_units_that_hold_do_not_drift(amq):
    """h of a constant input comes to rest at the input, however slowly.

    From 0 under a constant gate h_T = 1 - (1 - i)^T, which is 1 - 1.2e-3 here: the sequence is compared with that.  Every step rounds the
    state, the wave's factor and its offset by at most 2^-25 (values in [0.5, 1)); an error of d per step grows to d / i at rest."""
    T, n = 20000, 64
    gate = torch.full((T, 1, n), 8.0)
    hs, last, _ = amq.linear_recurrence(gate.to(DEV), torch.ones(T, 1, n).to(DEV))
    i = torch.sigmoid(torch.tensor(-8.0, dtype=torch.float64))
    want = -torch.expm1(T * torch.log1p(-i))
    assert abs(float(last[0, 0]) - float(want)) <= float(3 * 2.0 ** -25 / i) + 8 * U
    assert bool((last == last[0, 0]).all())


def test_a_nan_stays_in_its_channel_and_behind_its_step(amq):
    for T in (30, 300):
        gate, x, h0 = case(9, T, 2, 70, torch.float32, "blend")
        bad = x.clone()
        bad[T // 2, 1, 13] = float("nan")
        good = amq.linear_recurrence(gate.to(DEV), x.to(DEV), h0.to(DEV))[0].cpu()
        got = amq.linear_recurrence(gate.to(DEV), bad.to(DEV), h0.to(DEV))[0].cpu()
        assert bool(torch.isnan(got[T // 2:, 1, 13]).all())
        got[T // 2:, 1, 13] = good[T // 2:, 1, 13]
        assert torch.equal(got, good)


@pytest.mark.parametrize("T,B,n", [(30, 3, 70), (300, 3, 70), (3000, 3, 70), (300, 300, 70)])
@pytest.mark.parametrize("mode", MODES)
def test_padding_holds_what_an_entry_ends_in(amq, T, B, n, mode):
    """Also an infinity or NaN of its last step, in every form of the launch; its neighbours know nothing of it."""
    gate, x, h0 = case(10, T, B, n, torch.float32, mode)
    lengths = torch.tensor([T, max(1, T // 2), max(1, T // 2 - 3)]).repeat(B // 3 + 1)[:B]
    clean = amq.linear_recurrence(gate.to(DEV), x.to(DEV), h0.to(DEV), mode=mode, lengths=lengths.to(DEV))[1].cpu()
    bad = x.clone()
    for b in range(B):
        bad[lengths[b] - 1, b, 5] = float("inf")
        bad[lengths[b] - 1, b, 69] = float("nan")
    hs, last, _ = amq.linear_recurrence(gate.to(DEV), bad.to(DEV), h0.to(DEV), mode=mode, lengths=lengths.to(DEV))
    last, hs = last.cpu(), hs.cpu()
    assert bool((last[:, 5] == float("inf")).all()) and bool(torch.isnan(last[:, 69]).all())
    assert all(bool((hs[lengths[b]:, b] == 0).all()) for b in range(B))
    last[:, [5, 69]] = clean[:, [5, 69]]
    assert torch.equal(last, clean)


@pytest.mark.parametrize("mode", MODES)
def test_gradients_against_differences(amq, mode):
    """Central differences of the binary64 plain form; their own error is of order step^2."""
    T, B, n, step = 140, 1, 2, 1e-5
    gate, x, h0 = case(11, T, B, n, torch.float32, mode)
    dhs, dl = rand(21, T, B, n), rand(22, B, n)

    def loss(g, v, h):
        hs, _, _ = recurrence64(g, v, h, mode)
        return float((hs * dhs.double()).sum() + (hs[-1] * dl.double()).sum())

    states = amq.linear_recurrence(gate.to(DEV), x.to(DEV), h0.to(DEV), mode=mode, states=True)[2]
    got = amq.linear_recurrence_backward(dhs.to(DEV), gate.to(DEV), x.to(DEV), h0.to(DEV), states, dl.to(DEV), mode=mode)
    args = [t.double() for t in (gate, x, h0)]
    for i, places in ((0, [(0, 0, 0), (5, 0, 1), (127, 0, 0), (128, 0, 1), (139, 0, 0)]), (1, [(0, 0, 1), (64, 0, 0), (139, 0, 1)]), (2, [(0, 0), (0, 1)])):
        for at in places:
            side = []
            for sign in (1, -1):
                moved = [t.clone() for t in args]
                moved[i][at] += sign * step
                side.append(loss(*moved))
            want = (side[0] - side[1]) / (2 * step)
            assert abs(float(got[i][at]) - want) <= 1e-5 * (1 + abs(want)), (i, at)


def test_results_repeat(amq):
    gate, x, h0 = (t.to(DEV) for t in case(13, 3000, 2, 200, torch.bfloat16, "blend"))
    dhs, dl = rand(1, 3000, 2, 200).to(torch.bfloat16).to(DEV), rand(2, 2, 200).to(DEV)
    first = None
    for _ in range(5):
        hs, last, states = amq.linear_recurrence(gate, x, h0, states=True)
        got = (hs, last, states) + amq.linear_recurrence_backward(dhs, gate, x, h0, states, dl)
        assert first is None or all(torch.equal(p, q) for p, q in zip(got, first))
        first = got


def test_refusals(amq):
    gate, x, h0 = (t.to(DEV) for t in case(1, 200, 2, 6, torch.float32, "blend"))
    for bad in (dict(gate=gate[:1]), dict(gate=gate[0]), dict(h0=h0[:1]), dict(mode="other"), dict(states=None, backward=True), dict(dh_last=h0[:, :1], backward=True)):
        bad = dict(bad)
        back = bad.pop("backward", False)
        kw = dict(dict(gate=gate, x=x, h0=h0), **bad)
        with pytest.raises(ValueError):
            amq.linear_recurrence_backward(x, **kw) if back else amq.linear_recurrence(**kw)
    for bad in (dict(gate=gate.half()), dict(x=x.double()), dict(h0=h0.half()), dict(h0=h0.cpu()), dict(lengths=torch.zeros(2, dtype=torch.int32, device=DEV)),
                dict(out=x), dict(h_out=h0.half()), dict(gate=gate.transpose(1, 2).contiguous().transpose(1, 2)), dict(out=x[:1].expand_as(x).clone()[:, :1].expand_as(x))):
        with pytest.raises(amq.AmqError):
            amq.linear_recurrence(**dict(dict(gate=gate, x=x, h0=h0), **bad))
    for i in range(3):
        args = [gate, x, h0]
        args[i] = args[i].clone().requires_grad_()
        with pytest.raises(amq.AmqError, match="linear_recurrence"):
            amq.linear_recurrence(*args)
        with torch.no_grad():
            amq.linear_recurrence(*args)


@pytest.mark.parametrize("T,B,n", [(1, 2, 100), (35, 3, 50), (900, 1, 64)])
def test_captured(amq, T, B, n):
    """A step of serving with its state in place, and both passes, captured and replayed between eager calls."""
    gate, x, h0 = (t.to(DEV) for t in case(3, T, B, n, torch.bfloat16, "blend"))
    dhs = rand(4, T, B, n).to(torch.bfloat16).to(DEV)
    ws = amq.linear_recurrence_workspace(T, B, n, x.dtype, DEV)
    wsg = amq.linear_recurrence_backward_workspace(T, B, n, x.dtype, DEV)

    def both(g, v, h):
        hs, last, states = amq.linear_recurrence(g, v, h, states=True, ws=ws, h_out=h)
        return (hs,) + amq.linear_recurrence_backward(dhs, g, v, h, states, ws=wsg)

    h = h0.clone()
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        both(gate, x, h)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        out = both(gate, x, h)
    h.copy_(h0)
    state = h0.clone()
    for i in range(4):
        x.copy_(rand(20 + i, T, B, n))
        graph.replay()
        torch.cuda.synchronize()
        want = both(gate, x, state)
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(out, want)) and torch.equal(h, state), i


def test_another_stream(amq):
    gate, x, h0 = (t.to(DEV) for t in case(3, 500, 2, 64, torch.float32, "blend"))
    want = amq.linear_recurrence(gate, x, h0)[0]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(3)]
    got = []
    for s in streams:
        with torch.cuda.stream(s):
            got.append(amq.linear_recurrence(gate, x, h0)[0])
    torch.cuda.synchronize()
    assert all(torch.equal(g, want) for g in got)


def test_long_offsets(amq):
    """Entries whose offsets pass 32 bits: the last rows of a projection of 2^32 bytes and more."""
    T, n = 70, 64
    step = (1 << 26) + 2
    room = torch.zeros((T - 1) * step + 2 * n, dtype=torch.bfloat16, device=DEV)
    gate, x, h0 = case(3, T, 1, n, torch.bfloat16, "blend")
    g, v = room.as_strided((T, 1, n), (step, n, 1)), room.as_strided((T, 1, n), (step, n, 1), n)
    g.copy_(gate)
    v.copy_(x)
    check(amq, gate, x, h0, "blend", views=(g, v))
    check_grad(amq, gate, x, h0, "blend", views=(g, v))


@pytest.mark.parametrize("T,n", [((1 << 20) + 77, 2050), ((1 << 17) + 5, 17000)])
def test_more_than_32_bits_of_entries(amq, T, n):
    """Over 2^31 entries, with tiles in workgroups of their own and without: the sequence's end is that of its last steps alone, taken up from a state that
    the forward pass left; the backward pass's first steps are those of the beginning alone, with the gradient that reaches them.  (Two folds of
    the same maps in other places: the bound of the roundings behind that state.)"""
    g = torch.Generator(device=DEV).manual_seed(1)
    gate = torch.empty(T, 1, n, dtype=torch.bfloat16, device=DEV).normal_(generator=g)
    x = torch.empty_like(gate).normal_(generator=g)
    hs, last, states = amq.linear_recurrence(gate, x, states=True)
    at = (T - 1) // 128 * 128
    assert at * n > 1 << 31
    for view in ((gate[at - 128:], x[at - 128:], states[at // 128 - 2]),):
        tail, end, _ = amq.linear_recurrence(*view)
        ref, tol, _ = recurrence64(view[0].cpu().double(), view[1].cpu().double(), view[2].cpu().double(), "blend")
        assert_within(hs[at - 128:], ref, tol + half_ulp(torch.bfloat16) * ref.abs(), "hs")
        assert_within(last, ref[-1], tol[-1], "h_last")
    # the gradient of the last 300 steps' states, which reaches their beginning and no further than f decays
    dhs = torch.zeros_like(gate)
    dhs[-300:] = 1.0
    dgate, dx, dh0 = amq.linear_recurrence_backward(dhs, gate, x, torch.zeros(1, n, device=DEV), states)
    cut = at - 384
    tail = amq.linear_recurrence_backward(dhs[cut:], gate[cut:], x[cut:], states[cut // 128 - 1], amq.linear_recurrence(gate[cut:], x[cut:], states[cut // 128 - 1], states=True)[2])
    ref, tol = recurrence_grad64(dhs[cut:].cpu().double(), gate[cut:].cpu().double(), x[cut:].cpu().double(), states[cut // 128 - 1].cpu().double(),
                                 torch.zeros(1, n, dtype=torch.float64), "blend")
    for name, got, part, r, t in (("dgate", dgate, tail[0], ref[0], tol[0]), ("dx", dx, tail[1], ref[1], tol[1])):
        # (the gradient decays below 2^-126, the least normal number of either type, where no rounding is relative)
        t = t + half_ulp(torch.bfloat16) * r.abs() + 2.0 ** -126
        assert_within(got[cut:], r, t, name)
        assert_within(part, r, t, name + " of the part")
    assert bool((dx[:cut - 4000] == 0).all())


def test_many_at_once(amq):
    """Launches whose workgroups wait for each other, on several streams, more of them than the card holds."""
    cases = [[t.to(DEV) for t in case(i, 4000, 1, 512, torch.float32, "blend")] for i in range(4)]
    want = [amq.linear_recurrence(*c)[1] for c in cases]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in cases], []
    for _ in range(5):
        for s, c in zip(streams, cases):
            with torch.cuda.stream(s):
                got.append(amq.linear_recurrence(*c)[1])
    torch.cuda.synchronize()
    assert all(torch.equal(g, want[i % 4]) for i, g in enumerate(got))
