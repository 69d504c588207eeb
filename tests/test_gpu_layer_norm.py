"""Layer normalization, forward and backward, against the formulas in binary64.

Tolerances: between an entry and a result lie at most 96 roundings of binary32 (32 entries a lane, 16 waves, the
butterfly, and what follows), each of U times the magnitude of what is summed; 1.0 / sqrt and the statistics enter y
through (|x| + mean|x|) r |w|.  Column sums add up to `rows` terms.  Results are rounded once to their type.
"""
import pytest
import torch

from train_util import DEV, DTYPES, U, assert_within, half_ulp, rand, smallest

pytestmark = pytest.mark.gpu

# every form: a wave per row, four waves, sixteen, the general one; odd lengths, one entry, rows that share no alignment
SIZES = [(1, 1), (5, 3), (7, 64), (33, 129), (700, 300), (1030, 65), (2, 1024), (600, 2047), (3, 4097), (2, 8192), (2, 8193), (2, 16384),
         (3, 16385), (70, 20011)]


@pytest.fixture(scope="module")
def amq():
    import paper_1802_00150_amd as amq
    return amq


def case(seed, rows, n, dtype, params):
    x = (rand(seed, rows, n) * (0.5 + rand(seed + 1, n).abs()) + 0.5).to(dtype)
    return x, (1 + rand(seed + 2, n, scale=0.2)).to(params), rand(seed + 3, n, scale=0.2).to(params)


def stats64(x, eps):
    mean = x.mean(-1)
    var = ((x - mean[..., None]) ** 2).mean(-1)
    return mean, (var + eps) ** -0.5


def check_forward(got, x, w, b, eps, dtype, what):
    y, mean, rstd = got
    x, w, b = x.double(), w.double(), b.double()
    mean64, rstd64 = stats64(x, eps)
    ref = (x - mean64[..., None]) * rstd64[..., None] * w + b
    size = x.abs() + x.abs().mean(-1, keepdim=True)
    # where a row has no spread but eps, the error of the mean counts against sqrt(eps)
    tol = 96 * U * (2 * size * rstd64[..., None] * w.abs() + b.abs() + ref.abs()) + half_ulp(dtype) * ref.abs() + smallest(dtype)
    assert_within(y, ref, tol, what + " y")
    assert_within(mean, mean64, 96 * U * x.abs().mean(-1), what + " mean")
    assert_within(rstd, rstd64, 96 * U * rstd64 * (1 + rstd64 * x.abs().mean(-1)), what + " rstd")


@pytest.mark.parametrize("rows,n", SIZES)
@pytest.mark.parametrize("dtype", DTYPES)
def test_forward(amq, rows, n, dtype):
    x, w, b = case(rows + n, rows, n, dtype, torch.float32)
    check_forward(amq.layer_norm(x.to(DEV), w.to(DEV), b.to(DEV), 1e-5), x, w, b, 1e-5, dtype, "%dx%d" % (rows, n))


def check_backward(amq, rows, n, dtype, params, seed=0):
    x, w, _ = case(seed + rows + 3 * n, rows, n, dtype, params)
    dy = rand(seed + 9, rows, n).to(dtype)
    mean64, rstd64 = stats64(x.double(), 1e-5)
    mean, rstd = mean64.float(), rstd64.float()
    dx, dw, db = amq.layer_norm_backward(dy.to(DEV), x.to(DEV), w.to(DEV), mean.to(DEV), rstd.to(DEV))
    d, r = dy.double(), rstd.double()[:, None]
    z = (x.double() - mean.double()[:, None]) * r
    g = d * w.double()
    ref = r * (g - g.mean(1, keepdim=True) - z * (g * z).mean(1, keepdim=True))
    size = r * (g.abs() + g.abs().mean(1, keepdim=True) + z.abs() * (g * z).abs().mean(1, keepdim=True))
    # z itself is a difference of rounded values
    size = size + r * (x.double().abs() * r * (g * z).abs().mean(1, keepdim=True) + z.abs() * (g.abs() * x.double().abs() * r).mean(1, keepdim=True))
    assert_within(dx, ref, 96 * U * size + half_ulp(dtype) * ref.abs() + smallest(dtype), "dx")
    terms = 96 + rows
    ref = (d * z).sum(0)
    size = (d.abs() * (z.abs() + (x.double().abs() + mean.double().abs()[:, None]) * r)).sum(0)
    assert_within(dw, ref, terms * U * size + half_ulp(params) * ref.abs() + smallest(params), "dweight")
    assert_within(db, d.sum(0), terms * U * d.abs().sum(0) + half_ulp(params) * d.sum(0).abs() + smallest(params), "dbias")
    assert dw.dtype == db.dtype == params


@pytest.mark.parametrize("rows,n", SIZES)
@pytest.mark.parametrize("dtype", DTYPES)
def test_backward(amq, rows, n, dtype):
    if n == 1:
        pytest.skip("a row of one entry has no spread: tested with eps below")
    check_backward(amq, rows, n, dtype, torch.float32)


@pytest.mark.parametrize("dtype", DTYPES[1:])
def test_parameters_of_the_data_s_type(amq, dtype):
    x, w, b = case(3, 40, 200, dtype, dtype)
    check_forward(amq.layer_norm(x.to(DEV), w.to(DEV), b.to(DEV)), x, w, b, 1e-5, dtype, "params")
    check_backward(amq, 40, 200, dtype, dtype)


def test_more_rows_than_the_grid_takes_at_once(amq):
    check_backward(amq, 9001, 96, torch.float32, torch.float32)
    x, w, b = case(4, 20000, 40, torch.bfloat16, torch.float32)
    check_forward(amq.layer_norm(x.to(DEV), w.to(DEV), b.to(DEV)), x, w, b, 1e-5, torch.bfloat16, "many rows")


@pytest.mark.parametrize("dtype", DTYPES)
def test_rows_without_spread(amq, dtype):
    """Constant rows, rows of zeros and rows of one entry: eps alone is under the root, y is the bias."""
    for rows, n in ((4, 1), (3, 77), (2, 3000)):
        x = torch.full((rows, n), 0.75).to(dtype)
        x[0] = 0
        w, b = torch.full((n,), 2.0), rand(5, n)
        y, mean, rstd = amq.layer_norm(x.to(DEV), w.to(DEV), b.to(DEV), 1e-3)
        assert_within(mean, x.double().mean(1), 0.0, "mean")  # sums of 0.75 are exact
        assert_within(rstd, torch.full((rows,), 1e-3, dtype=torch.float64) ** -0.5, 4 * U * 32, "rstd")
        assert torch.equal(y.cpu(), b.to(dtype).expand(rows, n))
        dx, dw, db = amq.layer_norm_backward(torch.ones(rows, n, dtype=dtype, device=DEV), x.to(DEV), w.to(DEV), mean, rstd)
        # g = w is constant along the row: nothing is left of it but rounding
        assert_within(dx, torch.zeros(rows, n), 96 * U * 32 * 2, "dx")
        assert_within(dw, torch.zeros(n), 0.0, "dweight")
        assert_within(db, torch.full((n,), float(rows)), 0.0, "dbias")


def test_a_large_offset_does_not_swallow_the_variance(amq):
    x = (rand(6, 9, 500, scale=1e-2) + 100.0)
    check_forward(amq.layer_norm(x.to(DEV), torch.ones(500, device=DEV), torch.zeros(500, device=DEV)), x, torch.ones(500), torch.zeros(500),
                  1e-5, torch.float32, "offset")


@pytest.mark.parametrize("dtype", DTYPES)
def test_strides_offsets_and_in_place(amq, dtype):
    """Rows inside wider ones, beginning on any element; out = x; three dimensions."""
    for n, first, ld in ((61, 1, 70), (300, 3, 331), (1500, 5, 1511)):
        base = rand(7, 12, ld).to(dtype)
        x = base[:, first:first + n]
        w, b = 1 + rand(8, n, scale=0.1), rand(9, n)
        dev = base.to(DEV)
        xd = dev[:, first:first + n]
        y = amq.layer_norm(xd, w.to(DEV), b.to(DEV))[0]
        check_forward(amq.layer_norm(xd, w.to(DEV), b.to(DEV)), x, w, b, 1e-5, dtype, "strided")
        out, mean, rstd = amq.layer_norm(xd, w.to(DEV), b.to(DEV), out=xd)
        assert out is xd and torch.equal(xd, y)
        back = dev.cpu()
        assert torch.equal(back[:, :first], base[:, :first]) and torch.equal(back[:, first + n:], base[:, first + n:])
        dy = rand(10, 12, n).to(dtype).to(DEV)
        x2 = base.to(DEV)[:, first:first + n]
        one = amq.layer_norm_backward(dy, x2, w.to(DEV), mean, rstd)
        two = amq.layer_norm_backward(dy, x2, w.to(DEV), mean, rstd, out=dy)
        assert two[0] is dy and all(torch.equal(p, q) for p, q in zip(one, two))
    x = rand(11, 3, 4, 50).to(dtype).to(DEV)
    y, mean, rstd = amq.layer_norm(x)
    assert y.shape == x.shape and mean.shape == rstd.shape == (3, 4)
    assert torch.equal(y.view(12, 50), amq.layer_norm(x.view(12, 50))[0])


def test_without_parameters_or_their_gradients(amq):
    x, w, b = case(12, 20, 130, torch.float32, torch.float32)
    dy = rand(13, 20, 130).to(DEV)
    xd = x.to(DEV)
    y, mean, rstd = amq.layer_norm(xd)
    assert torch.equal(y, amq.layer_norm(xd, torch.ones(130, device=DEV), torch.zeros(130, device=DEV))[0])
    full = amq.layer_norm_backward(dy, xd, torch.ones(130, device=DEV), mean, rstd)
    assert all(torch.equal(p, q) for p, q in zip(full, amq.layer_norm_backward(dy, xd, None, mean, rstd)))
    dx, dw, db = amq.layer_norm_backward(dy, xd, None, mean, rstd, param_grads=False)
    assert dw is None and db is None and torch.equal(dx, full[0])


def test_same_results_every_time_and_on_another_stream(amq):
    x, w, b = case(14, 5000, 333, torch.bfloat16, torch.float32)
    xd, wd, bd, dy = x.to(DEV), w.to(DEV), b.to(DEV), rand(15, 5000, 333).to(torch.bfloat16).to(DEV)
    y, mean, rstd = amq.layer_norm(xd, wd, bd)
    first = amq.layer_norm_backward(dy, xd, wd, mean, rstd)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        y2, mean2, rstd2 = amq.layer_norm(xd, wd, bd)
        second = amq.layer_norm_backward(dy, xd, wd, mean2, rstd2)
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(y, y2) and all(torch.equal(p, q) for p, q in zip(first, second))


def test_gradient_against_differences(amq):
    """The autograd form: directional derivatives of a loss in binary64 against central differences.  A difference of
    losses with h = 1e-2 has an error of h^2 (third derivatives of order 1) and of rounding, 1e-7 / h: 1e-3 of the whole."""
    from paper_1802_00150_amd import training
    rows, n = 6, 40
    x, w, b, c = rand(16, rows, n), 1 + rand(17, n, scale=0.2), rand(18, n), rand(19, rows, n).double()
    leaves = [t.to(DEV).requires_grad_() for t in (x, w, b)]
    y = training.layer_norm(*leaves)
    y.backward(c.float().to(DEV))
    for i, leaf in enumerate(leaves):
        v = rand(20 + i, *leaf.shape).to(DEV)
        at = [t.detach() for t in leaves]

        def loss(t):
            moved = [a + t * v if j == i else a for j, a in enumerate(at)]
            return float((amq.layer_norm(*moved)[0].cpu().double() * c).sum())

        slope = (loss(1e-2) - loss(-1e-2)) / 2e-2
        mine = float((leaf.grad.double() * v.double()).sum())
        assert abs(slope - mine) <= 1e-3 * float((leaf.grad.double() * v.double()).abs().sum()), (i, slope, mine)


def test_refusals(amq):
    x, w = torch.zeros(4, 8, device=DEV), torch.ones(8, device=DEV)
    mean, rstd = torch.zeros(4, device=DEV), torch.ones(4, device=DEV)
    E = (amq.AmqError, ValueError)
    for bad in (lambda: amq.layer_norm(x.cpu()), lambda: amq.layer_norm(x.double()), lambda: amq.layer_norm(x[:0]),
                lambda: amq.layer_norm(x[:, :0]), lambda: amq.layer_norm(x.t()), lambda: amq.layer_norm(x[:1].expand(4, 8)),
                lambda: amq.layer_norm(x, w[:7]), lambda: amq.layer_norm(x, w.half()), lambda: amq.layer_norm(x, w, w.cpu()),
                lambda: amq.layer_norm(x, eps=-1.0), lambda: amq.layer_norm(x, out=torch.zeros(4, 7, device=DEV)),
                lambda: amq.layer_norm(x, out=x.half()), lambda: amq.layer_norm(x.half(), w, w.half()),
                lambda: amq.layer_norm_backward(x[:3], x, w, mean, rstd), lambda: amq.layer_norm_backward(x.half(), x, w, mean, rstd),
                lambda: amq.layer_norm_backward(x, x, w, mean[:3], rstd),
                lambda: amq.layer_norm_backward(x, x, w, mean, rstd, ws=torch.empty(16, dtype=torch.uint8, device=DEV))):
        with pytest.raises(E):
            bad()
