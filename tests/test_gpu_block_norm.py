"""Joined norms, forward and backward, against the formulas in binary64 (tolerances: recurrent_util)."""
import pytest
import torch

from recurrent_util import block_norm64, block_norm_grad64
from train_util import DEV, DTYPES, assert_within, half_ulp, rand, smallest

pytestmark = pytest.mark.gpu

# every form: rows of less than 16 bytes, a wave per row, four waves, eight, sixteen; odd lengths, rows that share no alignment, few and many rows
SIZES = [(1, 2), (5, 3), (3, 7), (9, 8), (7, 64), (33, 129), (700, 300), (1030, 65), (2, 512), (3, 513), (600, 513), (2, 1024), (515, 1024), (520, 1025),
         (600, 2047), (1, 16), (1300, 17), (70, 100), (2050, 128), (900, 130), (1111, 256), (3, 4097), (2, 8192), (3, 8193), (2, 16384)]
TYPES = [(torch.float32, torch.float32, torch.float32)] + [(t, r, p) for t in DTYPES[1:] for r in (t, torch.float32) for p in (t, torch.float32)]
EPS = 1e-5


@pytest.fixture(scope="module")
def amq():
    import paper_1802_00150_amd as amq
    return amq


def case(seed, rows, n, types, gate=True):
    dtype, residual, params = types
    x = (rand(seed, rows, n) * (0.5 + rand(seed + 1, n).abs()) + 0.5).to(dtype)
    h = rand(seed + 2, rows, n).to(residual)
    g = (rand(seed + 3, rows, n) * 2).to(dtype) if gate else None
    p = {"weight": 1 + rand(seed + 4, n, scale=0.2), "bias": rand(seed + 5, n, scale=0.2), "scale": 0.5 + rand(seed + 6, n, scale=0.2),
         "next_weight": 1 + rand(seed + 7, n, scale=0.2), "next_bias": rand(seed + 8, n, scale=0.2)}
    return x, h, g, {k: v.to(params) for k, v in p.items()}


def on(t):
    return None if t is None else t.to(DEV)


def full(p, n):
    """The parameters in binary64, absent ones as 1 and 0."""
    return [p[k].double() if p.get(k) is not None else torch.full((n,), float(k not in ("bias", "next_bias")), dtype=torch.float64)
            for k in ("weight", "bias", "scale", "next_weight", "next_bias")]


def within(got, ref, tol, what):
    t = got.dtype
    assert_within(got, ref, tol + half_ulp(t) * ref.abs() + smallest(t), what)


def check(amq, x, h, g, p, activation="sigmoid", what="", **kw):
    w, b, s, w2, b2 = full(p, x.shape[1])
    got = amq.block_norm(on(x), on(h), gate=on(g), activation=activation, eps=EPS, **{k: on(v) for k, v in p.items()}, **kw)
    ref, tol = block_norm64(x.double(), h.double(), w, b, None if g is None else g.double(), activation, s, w2, b2, EPS)
    assert got[0].dtype == h.dtype and got[1].dtype == x.dtype
    for name, q, r, t in zip(("y", "normed", "stats"), got, ref, tol):
        within(q, r, t, what + " " + name)
    return got


GRADS = ("dx", "dresidual", "dgate", "dweight", "dbias", "dscale", "dnext_weight", "dnext_bias")


def check_grad(amq, x, h, g, p, activation="sigmoid", dy=True, dn=True, what="", seed=0):
    rows, n = x.shape
    w, b, s, w2, b2 = full(p, n)
    gate = None if g is None else g.double()
    ref, _ = block_norm64(x.double(), h.double(), w, b, gate, activation, s, w2, b2, EPS)
    y, stats = ref[0].to(h.dtype), ref[2].float()
    dy = rand(seed + 20, rows, n).to(h.dtype) if dy else None
    dn = rand(seed + 21, rows, n).to(x.dtype) if dn else None
    got = amq.block_norm_backward(on(dy), on(dn), on(x), on(y), on(stats), gate=on(g), activation=activation, **{k: on(v) for k, v in p.items()})
    ref, tol = block_norm_grad64(None if dy is None else dy.double(), None if dn is None else dn.double(), x.double(), y.double(), stats.double(), w, b, gate,
                                 activation, s, w2)
    for name, q in zip(GRADS, got):
        if name == "dgate" and g is None or name[1:] in p and p[name[1:]] is None:
            assert q is None, name
            continue
        within(q, ref[name], tol[name], what + " " + name)
    return got


@pytest.mark.parametrize("rows,n", SIZES)
@pytest.mark.parametrize("types", TYPES[:1] + TYPES[2:3] + TYPES[4:5] + TYPES[8:9])
def test_sizes(amq, rows, n, types):
    x, h, g, p = case(rows + n, rows, n, types)
    check(amq, x, h, g, p, what="%dx%d" % (rows, n))
    check_grad(amq, x, h, g, p, what="%dx%d" % (rows, n))


@pytest.mark.parametrize("types", TYPES)
def test_types(amq, types):
    for rows, n in ((40, 200), (6, 3000)):
        x, h, g, p = case(rows, rows, n, types)
        check(amq, x, h, g, p)
        got = check_grad(amq, x, h, g, p)
        assert [t.dtype for t in got] == [types[0], types[1], types[0]] + [types[2]] * 5


@pytest.mark.parametrize("activation", [None, "none", "sigmoid", "silu"])
@pytest.mark.parametrize("gate", [False, True])
@pytest.mark.parametrize("types", [TYPES[0], TYPES[2]])
def test_gates(amq, activation, gate, types):
    x, h, g, p = case(3, 37, 130, types, gate)
    check(amq, x, h, g, p, activation)
    check_grad(amq, x, h, g, p, activation)


@pytest.mark.parametrize("absent", [("weight",), ("bias",), ("scale",), ("next_weight",), ("next_bias",), ("weight", "bias", "scale", "next_weight", "next_bias")])
@pytest.mark.parametrize("types", [TYPES[0], TYPES[1]])
def test_absent_parameters(amq, absent, types):
    x, h, g, p = case(4, 21, 90, types)
    p.update({k: None for k in absent})
    check(amq, x, h, g, p)
    check_grad(amq, x, h, g, p)


@pytest.mark.parametrize("n", [5, 300, 1500, 5000])
@pytest.mark.parametrize("types", [TYPES[0], TYPES[2]])
def test_one_gradient_alone(amq, n, types):
    """dy or dnormed None are zeros; without param_grads the others are the same."""
    x, h, g, p = case(5, 19, n, types)
    check_grad(amq, x, h, g, p, dy=False)
    check_grad(amq, x, h, g, p, dn=False)
    y, normed, stats = amq.block_norm(on(x), on(h), gate=on(g), **{k: on(v) for k, v in p.items()})
    args = on(rand(1, 19, n).to(h.dtype)), on(rand(2, 19, n).to(x.dtype)), on(x), y, stats
    kw = dict(gate=on(g), **{k: on(v) for k, v in p.items()})
    every, some = amq.block_norm_backward(*args, **kw), amq.block_norm_backward(*args, param_grads=False, **kw)
    assert all(torch.equal(a, b) for a, b in zip(every[:3], some[:3])) and some[3:] == (None,) * 5


@pytest.mark.parametrize("types", [TYPES[0], TYPES[2]])
def test_without_the_second_norm(amq, types):
    x, h, g, p = case(6, 30, 700, types)
    kw = dict(gate=on(g), **{k: on(p[k]) for k in ("weight", "bias", "scale")})
    y, normed, stats = amq.block_norm(on(x), on(h), **kw)
    y1, none, stats1 = amq.block_norm(on(x), on(h), normed=False, **kw)
    assert none is None and torch.equal(y, y1) and torch.equal(stats[:2], stats1[:2])
    dy = on(rand(1, 30, 700).to(h.dtype))
    a = amq.block_norm_backward(dy, None, on(x), y, stats1, **kw)
    b = amq.block_norm_backward(dy, None, on(x), y, stats, **kw)
    assert all(p is q is None or torch.equal(p, q) for p, q in zip(a, b))


def test_more_rows_than_the_grid_takes_at_once(amq):
    for rows, n, types in ((9001, 96, TYPES[0]), (20000, 40, TYPES[2]), (2600, 1200, TYPES[1]), (3000, 5, TYPES[8])):
        x, h, g, p = case(7, rows, n, types)
        check(amq, x, h, g, p)
        check_grad(amq, x, h, g, p)


@pytest.mark.parametrize("n", [3, 65, 700, 3001])
@pytest.mark.parametrize("types", [TYPES[0], TYPES[1], TYPES[2]])
def test_strides_and_places(amq, n, types):
    """Columns of wider matrices at odd offsets; y over the residual."""
    x, h, g, p = case(8, 23, n, types)
    want = amq.block_norm(on(x), on(h), gate=on(g), **{k: on(v) for k, v in p.items()})
    wide, tall = torch.full((23, 3 * n + 5), 7.0, dtype=x.dtype, device=DEV), torch.full((23, 2 * n + 3), 7.0, dtype=h.dtype, device=DEV)
    a, b, c = wide[:, 1:n + 1], wide[:, n + 2:2 * n + 2], wide[:, 2 * n + 3:3 * n + 3]
    a.copy_(x), b.copy_(g)
    hs, ys = tall[:, :n], tall[:, n + 1:2 * n + 1]
    hs.copy_(h)
    params = {k: on(v) for k, v in p.items()}
    got = amq.block_norm(a, hs, gate=b, out=ys, out_normed=c, **params)
    assert got[0] is ys and got[1] is c and all(torch.equal(u, v) for u, v in zip(got, want))
    assert bool((wide[:, 0] == 7).all() and (wide[:, n + 1] == 7).all() and (wide[:, 2 * n + 2] == 7).all() and (tall[:, n] == 7).all() and (tall[:, -1] == 7).all())
    got = amq.block_norm(a, hs, gate=b, out=hs, **params)
    assert got[0] is hs and all(torch.equal(u, v) for u, v in zip(got, want))
    dy, dn = on(rand(1, 23, n).to(h.dtype)), on(rand(2, 23, n).to(x.dtype))
    plain = amq.block_norm_backward(dy, dn, on(x), want[0], want[2], gate=on(g), **params)
    c.copy_(dn)
    strided = amq.block_norm_backward(dy, c, a, ys, want[2], gate=b, **params)
    assert all(torch.equal(u, v) for u, v in zip(plain, strided))


def test_more_dimensions(amq):
    x, h, g, p = case(9, 12, 60, TYPES[2])
    params = {k: on(v) for k, v in p.items()}
    want = amq.block_norm(on(x), on(h), gate=on(g), **params)
    got = amq.block_norm(on(x).view(3, 4, 60), on(h).view(3, 4, 60), gate=on(g).view(3, 4, 60), **params)
    assert got[0].shape == got[1].shape == (3, 4, 60) and all(torch.equal(a.reshape(b.shape), b) for a, b in zip(got, want))


@pytest.mark.parametrize("types", [TYPES[0], TYPES[2]])
def test_rows_without_spread(amq, types):
    """Constant rows: eps alone is under the root."""
    x, h, g, p = case(10, 6, 77, types)
    x.fill_(0.75), x[0].zero_()
    h[1].zero_()
    check(amq, x, h, g, p)
    p["scale"].zero_()
    h.fill_(0.5)
    check(amq, x, h, g, p)


def test_large_gates(amq):
    """Gates at which the exponential leaves its range."""
    x, h, _, p = case(11, 5, 8, TYPES[0])
    g = torch.tensor([float("inf"), 200.0, 100.0, 89.0, -89.0, -100.0, -200.0, 0.0]).repeat(5, 1)
    for activation in ("sigmoid", "silu"):
        if activation == "silu":
            g[:, 0] = 1000.0
        y, n, stats = amq.block_norm(on(x), on(h), gate=on(g), activation=activation, **{k: on(v) for k, v in p.items()})
        assert bool(torch.isfinite(y).all() and torch.isfinite(n).all())
        got = amq.block_norm_backward(on(h), on(x), on(x), y, stats, gate=on(g), activation=activation, **{k: on(v) for k, v in p.items()})
        assert all(bool(torch.isfinite(t).all()) for t in got)
        assert torch.equal(y.cpu()[:, 6], h[:, 6])


def test_gradients_against_differences(amq):
    """Central differences of the binary64 plain form at some entries; their own error is of order step^2."""
    rows, n, step = 3, 12, 1e-5
    for activation in ("sigmoid", "silu", None):
        x, h, g, p = case(12, rows, n, TYPES[0])
        dy, dn = rand(1, rows, n), rand(2, rows, n)
        names = ["weight", "bias", "scale", "next_weight", "next_bias"]
        leaves = [x.double(), h.double(), g.double()] + [p[k].double() for k in names]

        def loss(v):
            (y, m, _), _ = block_norm64(v[0], v[1], v[3], v[4], v[2], activation, v[5], v[6], v[7], EPS)
            return float((y * dy.double()).sum() + (m * dn.double()).sum())

        y, _, stats = amq.block_norm(on(x), on(h), gate=on(g), activation=activation, **{k: on(v) for k, v in p.items()})
        got = amq.block_norm_backward(on(dy), on(dn), on(x), y, stats, gate=on(g), activation=activation, **{k: on(v) for k, v in p.items()})
        for i, t in enumerate(got):
            for at in ((0, 0), (1, 5), (2, 11)) if t.dim() == 2 else ((0,), (7,)):
                side = []
                for sign in (1, -1):
                    moved = [v.clone() for v in leaves]
                    moved[i][at] += sign * step
                    side.append(loss(moved))
                want = (side[0] - side[1]) / (2 * step)
                assert abs(float(t[at]) - want) <= 1e-5 * (1 + abs(want)), (activation, GRADS[i], at)


def test_refusals(amq):
    x, h, g, p = case(13, 6, 20, TYPES[2])
    x, h, g, p = on(x), on(h), on(g), {k: on(v) for k, v in p.items()}
    for bad in (dict(residual=h[:5]), dict(gate=g[:, :10]), dict(weight=p["weight"][:5]), dict(activation="relu"), dict(normed=False, next_weight=p["next_weight"])):
        with pytest.raises(ValueError):
            amq.block_norm(**dict(dict(x=x, residual=h, gate=g), **bad))
    for bad in (dict(x=x.double()), dict(residual=h.half()), dict(gate=g.float()), dict(scale=p["scale"].bfloat16(), weight=p["weight"].float()), dict(weight=p["weight"].half()),
                dict(residual=h.cpu()), dict(out=x.float()[:, :20].expand(6, 20)[:1].expand(6, 20))):
        with pytest.raises(amq.AmqError):
            amq.block_norm(**dict(dict(x=x, residual=h, gate=g), **bad))
    for key, t in dict(p, x=x, residual=h, gate=g).items():
        kw = dict(dict(p, x=x, residual=h, gate=g), **{key: t.clone().requires_grad_()})
        with pytest.raises(amq.AmqError, match="block_norm"):
            amq.block_norm(**kw)
        with torch.no_grad():
            amq.block_norm(**kw)
    y, n, stats = amq.block_norm(x, h)
    for bad in (dict(dy=None, dnormed=None), dict(stats=stats[:2]), dict(y=y[:3])):
        with pytest.raises(ValueError):
            amq.block_norm_backward(**dict(dict(dy=y, dnormed=n, x=x, y=y, stats=stats), **bad))


def test_captured(amq):
    x, h, g, p = case(14, 300, 650, TYPES[2])
    x, h, g, p = on(x), on(h), on(g), {k: on(v) for k, v in p.items()}
    dy, dn = on(rand(1, 300, 650).to(h.dtype)), on(rand(2, 300, 650).to(x.dtype))
    ws = amq.block_norm_backward_workspace(300, 650, DEV)

    def both():
        y, n, stats = amq.block_norm(x, h, gate=g, activation="silu", **p)
        return (y, n, stats) + amq.block_norm_backward(dy, dn, x, y, stats, gate=g, activation="silu", ws=ws, **p)

    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        both()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        out = both()
    for i in range(4):
        x.copy_(rand(20 + i, 300, 650))
        graph.replay()
        torch.cuda.synchronize()
        want = both()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want)), i


def test_long_offsets(amq):
    """Rows whose offsets pass 32 bits."""
    x, h, g, p = case(15, 70, 66, TYPES[2])
    params = {k: on(v) for k, v in p.items()}
    step = (1 << 26) + 6
    room = torch.zeros(69 * step + 5 * 66, dtype=x.dtype, device=DEV)
    a, b, c, d, e = (room.as_strided((70, 66), (step, 1), i * 66) for i in range(5))
    a.copy_(x), b.copy_(h), c.copy_(g)
    want = amq.block_norm(on(x), on(h), gate=on(g), **params)
    got = amq.block_norm(a, b, gate=c, out=d, out_normed=e, **params)
    assert all(torch.equal(u, v) for u, v in zip(got, want))
    dy, dn = on(rand(1, 70, 66).to(h.dtype)), on(rand(2, 70, 66).to(x.dtype))
    plain = amq.block_norm_backward(dy, dn, on(x), want[0], want[2], gate=on(g), **params)
    far = amq.block_norm_backward(dy, dn, a, d, want[2], gate=c, **params)
    assert all(torch.equal(u, v) for u, v in zip(plain, far))
