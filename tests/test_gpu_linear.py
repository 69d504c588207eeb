"""Linear layers with their epilogue, forward and backward, against the formulas in binary64.

Tolerances, per element: a sum of k products accumulated in binary32 errs by at most (k + 16) U sum |a||b|; float operands
are split into 22 bits, 2^-21 sum |a||b|; activations have slopes of at most 1.2 and errors of their own of 8 U; results are
rounded once.  With an activation, d of the backward pass is rounded to the type in between.  Since those are worst cases
over k terms, the 2-norm is held to what independent roundings leave.
"""
import pytest
import torch

from train_util import ACTS, DEV, DTYPES, U, act64, assert_within, half_ulp, rand, relative, slope64, smallest

pytestmark = pytest.mark.gpu

# few rows (up to 8); one tile; split contractions; tiles of 64, 128 and 256; sizes that are no multiple of anything
SIZES = [(1, 1, 1), (1, 1024, 1024), (2, 7, 5), (4, 130, 33), (8, 301, 66), (9, 1, 1), (9, 63, 65), (17, 64, 64), (64, 1024, 128), (100, 2000, 70),
         (129, 200, 515), (300, 65, 300)]
LARGE = [(2300, 200, 1800), (3600, 130, 4100)]


@pytest.fixture(scope="module")
def amq():
    import paper_1802_00150_amd as amq
    return amq


def split_error(dtype):
    return 2.0 ** -21 if dtype == torch.float32 else 0.0


def norm_bound(dtype, roundings=1):
    """Relative 2-norm of results: `roundings` independent ones to the type (each half_ulp at most), or the errors of
    binary32 sums and split operands, 2^-22 a term."""
    return 1e-6 if dtype == torch.float32 else half_ulp(dtype) * roundings ** 0.5


def inputs(seed, rows, k, n, dtype):
    return (rand(seed, rows, k).to(dtype), rand(seed + 1, n, k, scale=k ** -0.5).to(dtype), rand(seed + 2, n, scale=0.5).to(dtype),
            rand(seed + 3, rows, n).to(dtype))


def check_forward(amq, rows, k, n, dtype, act, seed=0, bias=True, residual=True):
    x, W, b, r = inputs(seed + rows + k + n, rows, k, n, dtype)
    pre = torch.empty(rows, n, dtype=dtype, device=DEV)
    y = amq.linear(x.to(DEV), W.to(DEV), b.to(DEV) if bias else None, act, r.to(DEV) if residual else None, pre=pre)
    z = x.double() @ W.double().t() + (b.double() if bias else 0)
    size = x.double().abs() @ W.double().abs().t() + (b.double().abs() if bias else 0)
    err = ((k + 16) * U + split_error(dtype)) * size
    assert_within(pre, z, err + half_ulp(dtype) * z.abs() + smallest(dtype), "pre")
    ref = act64(z, act) + (r.double() if residual else 0)
    tol = 1.2 * err + 8 * U * (1 + z.abs()) + half_ulp(dtype) * ref.abs() * 1.01 + smallest(dtype)
    assert_within(y, ref, tol, "y")
    assert relative(pre, z) <= norm_bound(dtype)


@pytest.mark.parametrize("rows,k,n", SIZES)
@pytest.mark.parametrize("dtype", DTYPES)
def test_forward(amq, rows, k, n, dtype):
    check_forward(amq, rows, k, n, dtype, ACTS[(rows + k + n) % 6])


@pytest.mark.parametrize("k,n", [(2048, 2056), (1000, 3000), (999, 1501), (24, 40)])
@pytest.mark.parametrize("rows", [1, 2, 4, 5, 8])
@pytest.mark.parametrize("dtype", DTYPES)
def test_few_rows(amq, rows, k, n, dtype):
    """On either side of the choice between the vector units and the matrix cores; the caller's workspace too."""
    check_forward(amq, rows, k, n, dtype, "silu")
    x, W, b, r = (t.to(DEV) for t in inputs(rows, rows, k, n, dtype))
    y = amq.linear(x, W, b, None, r)
    assert torch.equal(y, amq.linear(x, W, b, None, r, ws=amq.linear_workspace(rows, k, n, dtype, DEV).fill_(0xFF)))


@pytest.mark.parametrize("rows,k,n", LARGE)
@pytest.mark.parametrize("dtype", DTYPES)
def test_forward_large_tiles(amq, rows, k, n, dtype):
    check_forward(amq, rows, k, n, dtype, "gelu")


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("dtype", DTYPES)
def test_every_activation(amq, act, dtype):
    check_forward(amq, 3, 40, 50, dtype, act, bias=False)
    check_forward(amq, 70, 40, 50, dtype, act, residual=False)
    check_backward(amq, 70, 40, 50, dtype, act)


def check_backward(amq, rows, k, n, dtype, act, seed=0):
    x, W, b, dy = inputs(seed + rows + k + n, rows, k, n, dtype)
    pre = (x.double() @ W.double().t() + b.double()).to(dtype) if act != "none" else None
    dx, dW, db = amq.linear_backward(dy.to(DEV), x.to(DEV), W.to(DEV), None if pre is None else pre.to(DEV), act)
    d = dy.double() if pre is None else dy.double() * slope64(pre.double(), act)
    # slopes err by 8 U of 1 + z^2 at most; then d is rounded
    d_err = torch.zeros_like(d) if pre is None else dy.double().abs() * 8 * U * (1 + pre.double() ** 2) + half_ulp(dtype) * d.abs()
    if pre is not None and dtype == torch.float16:
        d_err = d_err + 2.0 ** -38 * d.abs().max()
    for got, ref, size, err, terms, what in (
            (dx, d @ W.double(), d.abs() @ W.double().abs(), d_err @ W.double().abs(), n, "dx"),
            (dW, d.t() @ x.double(), d.abs().t() @ x.double().abs(), d_err.t() @ x.double().abs(), rows, "dW"),
            (db, d.sum(0), d.abs().sum(0), torch.zeros(n, dtype=torch.float64) if pre is None else (dy.double().abs() * 8 * U * (1 + pre.double() ** 2)).sum(0), rows,
             "dbias")):
        tol = ((terms + 16) * U + split_error(dtype)) * size + err * 1.01 + half_ulp(dtype) * ref.abs() * 1.01 + smallest(dtype)
        assert_within(got, ref, tol, what)
        if ref.numel() >= 4096:
            assert relative(got, ref) <= norm_bound(dtype, 1 if pre is None else 2), what


@pytest.mark.parametrize("rows,k,n", SIZES)
@pytest.mark.parametrize("dtype", DTYPES)
def test_backward(amq, rows, k, n, dtype):
    check_backward(amq, rows, k, n, dtype, ACTS[(rows + k + n) % 6])


@pytest.mark.parametrize("rows,k,n", LARGE)
@pytest.mark.parametrize("dtype", DTYPES)
def test_backward_large_tiles(amq, rows, k, n, dtype):
    check_backward(amq, rows, k, n, dtype, "silu")


@pytest.mark.parametrize("dtype", DTYPES)
def test_strides_offsets_and_in_place(amq, dtype):
    """Operands inside wider tensors, beginning on any element; the result over the residual; three dimensions."""
    for rows, k, n in ((5, 70, 33), (90, 128, 64), (90, 100, 61)):
        x, W, b, r = (t.to(DEV) for t in inputs(1, rows, k, n, dtype))
        plain = amq.linear(x, W, b, "silu", r)

        def inside(t, first, extra):
            wide = torch.full((t.shape[0], t.shape[1] + extra), float("nan"), dtype=dtype, device=DEV)
            wide[:, first:first + t.shape[1]] = t
            return wide, wide[:, first:first + t.shape[1]]

        (_, xs), (_, Ws), (wide, rs) = inside(x, 1, 5), inside(W, 3, 9), inside(r, 1, 3)
        y = amq.linear(xs, Ws, b, "silu", rs, out=rs)
        assert y is rs and torch.equal(rs, plain)
        assert torch.isnan(wide[:, :1]).all() and torch.isnan(wide[:, 1 + n:]).all()
        dy, pre = rand(5, rows, n).to(dtype).to(DEV), torch.empty(rows, n, dtype=dtype, device=DEV)
        amq.linear(x, W, b, "silu", pre=pre)
        one = amq.linear_backward(dy, x, W, pre, "silu")
        two = amq.linear_backward(inside(dy, 1, 2)[1], xs, Ws, inside(pre, 2, 5)[1], "silu")
        assert all(torch.equal(p, q) for p, q in zip(one, two))
    x, W, b, r = (t.to(DEV) for t in inputs(2, 24, 64, 40, dtype))
    assert torch.equal(amq.linear(x.view(2, 3, 4, 64), W, b, None, r.view(2, 3, 4, 40)).view(24, 40), amq.linear(x, W, b, None, r))


def test_any_subset_of_the_gradients(amq):
    x, W, b, dy = (t.to(DEV) for t in inputs(3, 50, 60, 70, torch.float32))
    pre = amq.linear(x, W, b)
    full = amq.linear_backward(dy, x, W, pre, "tanh")
    for i in range(1, 8):
        got = amq.linear_backward(dy, x, W, pre, "tanh", bool(i & 1), bool(i & 2), bool(i & 4))
        for j in range(3):
            assert (got[j] is None) == (not i >> j & 1)
            assert got[j] is None or torch.equal(got[j], full[j])


@pytest.mark.parametrize("rows,k,n", [(40, 96, 72), (1200, 640, 1300)])
def test_rows_of_unlike_scale(amq, rows, k, n):
    """Float rows 2^60 apart, entries 2^24 apart within one, rows of zeros, subnormal rows: the scale is each row's own.
    (Few numbers are multiplied in binary32, many as split ones.)"""
    x, W = rand(4, rows, k), rand(5, n, k)
    x *= 2.0 ** (torch.arange(rows) % 7 * 20 - 60)[:, None]
    x[:, ::3] *= 2.0 ** -24
    x[3] = 0
    x[4] = rand(6, k) * 2.0 ** -135
    W *= 2.0 ** (torch.arange(n) % 5 * 10 - 20)[:, None]
    W[7] = 0
    y = amq.linear(x.to(DEV), W.to(DEV))
    ref = x.double() @ W.double().t()
    size = x.double().abs() @ W.double().abs().t()
    assert_within(y, ref, ((k + 16) * U + 2.0 ** -21) * size + 2.0 ** -149, "y")
    dy = rand(7, rows, n) * 2.0 ** (torch.arange(n) % 9 * 12 - 48)
    dx, dW, db = amq.linear_backward(dy.to(DEV), x.to(DEV), W.to(DEV))
    # an operand's smallest step is 2^-38 of its row's largest entry
    step = 2.0 ** -38
    for got, a, c, terms, what in ((dx, dy, W.t(), n, "dx"), (dW, dy.t(), x.t(), rows, "dW")):
        a, c = a.double(), c.double()
        tol = ((terms + 16) * U + 2.0 ** -21) * (a.abs() @ c.abs().t())
        tol += step * (a.abs().sum(1)[:, None] * c.abs().amax(1)[None] + a.abs().amax(1)[:, None] * c.abs().sum(1)[None]) + 2.0 ** -149
        assert_within(got, a @ c.t(), tol, what)


def test_small_half_gradients_keep_their_digits(amq):
    """dy = 1e-4 and below, where half has few digits: d is scaled before it is rounded."""
    rows, k, n = 512, 128, 192
    x, W, b, _ = inputs(8, rows, k, n, torch.float16)
    pre = (x.double() @ W.double().t()).half()
    dy = rand(9, rows, n, scale=1e-4).half()
    dx, dW, db = amq.linear_backward(dy.to(DEV), x.to(DEV), W.to(DEV), pre.to(DEV), "sigmoid")
    d = dy.double() * slope64(pre.double(), "sigmoid")
    ref = d.t() @ x.double()
    assert relative(dW, ref) <= norm_bound(torch.float16, 2) + smallest(torch.float16) / float(ref.square().mean().sqrt())


@pytest.mark.parametrize("bad", [float("inf"), float("-inf"), float("nan")])
@pytest.mark.parametrize("dtype", DTYPES)
def test_infinities_and_nan_stay_where_they_enter(amq, bad, dtype):
    """One entry of x, of W and of dy: results that do not depend on it are those of a zero in its place, bit for bit; the
    others are not finite."""
    for rows, k, n in ((5, 70, 33), (150, 90, 130)):
        x, W, b, dy = (t.to(DEV) for t in inputs(14, rows, k, n, dtype))
        pre = amq.linear(x, W, b)

        def with_entry(t, i, j, v):
            t = t.clone()
            t[i, j] = v
            return t

        def same_but(got, ref, spoiled):
            assert torch.equal(got[~spoiled], ref[~spoiled]) and not torch.isfinite(got[spoiled]).any()

        def line(t, row=None, col=None):
            m = torch.zeros(t.shape, dtype=torch.bool, device=DEV)
            m[(row if row is not None else slice(None), col if col is not None else slice(None))] = True
            return m

        y = [amq.linear(with_entry(x, 3, 7, v), W, b) for v in (bad, 0.0)]
        same_but(*y, line(y[0], row=3))
        y = [amq.linear(x, with_entry(W, 4, 6, v), b) for v in (bad, 0.0)]
        same_but(*y, line(y[0], col=4))
        for act in (None, "sigmoid"):
            got, ref = (amq.linear_backward(with_entry(dy, 2, 5, v), x, W, pre, act) for v in (bad, 0.0))
            same_but(got[0], ref[0], line(got[0], row=2))
            same_but(got[1], ref[1], line(got[1], row=5))
            assert torch.equal(got[2][:5], ref[2][:5]) and torch.equal(got[2][6:], ref[2][6:]) and not torch.isfinite(got[2][5])
            got, ref = (amq.linear_backward(dy, with_entry(x, 3, 7, v), with_entry(W, 4, 6, v), pre, act) for v in (bad, 0.0))
            same_but(got[0], ref[0], line(got[0], col=6))
            same_but(got[1], ref[1], line(got[1], col=7))


def test_workspaces_streams_and_repeats(amq):
    """The caller's workspace with anything in it; another stream; the same results every time."""
    for dtype in DTYPES:
        for rows, k, n in ((3, 50, 60), (70, 50, 60), (64, 2048, 64)):
            x, W, b, dy = (t.to(DEV) for t in inputs(10, rows, k, n, dtype))
            y = amq.linear(x, W, b, "gelu")
            pre = amq.linear(x, W, b)
            back = amq.linear_backward(dy, x, W, pre, "gelu")
            ws = amq.linear_workspace(rows, k, n, dtype, DEV).fill_(0xFF)
            wb = amq.linear_backward_workspace(rows, k, n, dtype, DEV).fill_(0xFF)
            s = torch.cuda.Stream()
            s.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(s):
                y2 = amq.linear(x, W, b, "gelu", ws=ws)
                back2 = amq.linear_backward(dy, x, W, pre, "gelu", ws=wb)
            torch.cuda.current_stream().wait_stream(s)
            assert torch.equal(y, y2) and all(torch.equal(p, q) for p, q in zip(back, back2))


def test_graph_replays(amq):
    x, W, b, dy = (t.to(DEV) for t in inputs(11, 70, 100, 90, torch.float32))
    pre, out = torch.empty(70, 90, device=DEV), torch.empty(70, 90, device=DEV)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        amq.linear(x, W, b, "silu", out=out, pre=pre)
        amq.linear_backward(dy, x, W, pre, "silu")
    torch.cuda.current_stream().wait_stream(s)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        amq.linear(x, W, b, "silu", out=out, pre=pre)
        grads = amq.linear_backward(dy, x, W, pre, "silu")
    for i in range(3):
        x.copy_(rand(20 + i, 70, 100))
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        p = torch.empty_like(pre)
        assert torch.equal(out, amq.linear(x, W, b, "silu", pre=p))
        assert all(torch.equal(a, c) for a, c in zip(grads, amq.linear_backward(dy, x, W, p, "silu")))


def test_gradient_against_differences(amq):
    """The autograd form: directional derivatives against central differences (h = 1e-2: h^2, and rounding 1e-7 / h)."""
    from paper_1802_00150_amd import training
    x, W, b, r = inputs(12, 20, 30, 25, torch.float32)
    c = rand(13, 20, 25).double()
    for act in ("gelu", "silu", "sigmoid", "tanh", None):
        leaves = [t.to(DEV).requires_grad_() for t in (x, W, b, r)]
        training.linear(leaves[0], leaves[1], leaves[2], act, leaves[3]).backward(c.float().to(DEV))
        for i, leaf in enumerate(leaves):
            v = rand(30 + i, *leaf.shape).to(DEV)
            at = [t.detach() for t in leaves]

            def loss(t):
                m = [a + t * v if j == i else a for j, a in enumerate(at)]
                return float((amq.linear(m[0], m[1], m[2], act, m[3]).cpu().double() * c).sum())

            slope, mine = (loss(1e-2) - loss(-1e-2)) / 2e-2, float((leaf.grad.double() * v.double()).sum())
            assert abs(slope - mine) <= 1e-3 * float((leaf.grad.double() * v.double()).abs().sum()), (act, i, slope, mine)


def test_refusals(amq):
    x, W, b = torch.zeros(4, 8, device=DEV), torch.zeros(5, 8, device=DEV), torch.zeros(5, device=DEV)
    dy = torch.zeros(4, 5, device=DEV)
    small = torch.empty(16, dtype=torch.uint8, device=DEV)
    x9 = torch.zeros(9, 8, device=DEV)
    for bad in (lambda: amq.linear(x.cpu(), W), lambda: amq.linear(x, W.cpu()), lambda: amq.linear(x, W.half()), lambda: amq.linear(x.double(), W.double()),
                lambda: amq.linear(x, W[:, :7]), lambda: amq.linear(x, W, b[:4]), lambda: amq.linear(x, W, b.half()), lambda: amq.linear(x, W, b, "swish"),
                lambda: amq.linear(x, W, b, None, dy[:3]), lambda: amq.linear(x[:0], W), lambda: amq.linear(x, W[:0]), lambda: amq.linear(x.t(), W),
                lambda: amq.linear(x, W, out=torch.zeros(4, 6, device=DEV)), lambda: amq.linear(x, W, pre=torch.zeros(4, 4, device=DEV)),
                lambda: amq.linear(x9, W, ws=small),
                lambda: amq.linear_backward(dy, x, W, None, "relu"), lambda: amq.linear_backward(dy[:, :4], x, W),
                lambda: amq.linear_backward(dy, x, W, input_grad=False, weight_grad=False, bias=False),
                lambda: amq.linear_backward(dy, x, W, ws=small)):
        with pytest.raises((amq.AmqError, ValueError)):
            bad()
