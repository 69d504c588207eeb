"""Layer normalization of rows outside the range whose entries a wave or workgroup holds: of more than 16384 entries, and of less than 16 bytes.

Tolerances are those of the other layer norm tests.
"""
import pytest
import torch

from train_util import DEV, DTYPES, U, half_ulp, rand, smallest
from test_gpu_layer_norm import case, check_backward, check_forward

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def amq():
    import paper_1802_00150_amd as amq
    return amq


# (the forms for 16 bytes and more beside them: with four waves per row, with one, with sixteen)
@pytest.mark.parametrize("n", [3, 7, 8, 301, 1500, 16384, 16385, 20011])
@pytest.mark.parametrize("dtype", DTYPES)
def test_backward_in_place(amq, n, dtype):
    """dx over dy or over x: all three gradients are those of a dx of its own."""
    for rows in (5, 70, 300):
        x, w, _ = case(rows + n, rows, n, dtype, torch.float32)
        x, w, dy = x.to(DEV), w.to(DEV), rand(1, rows, n).to(dtype).to(DEV)
        _, mean, rstd = amq.layer_norm(x)
        apart = amq.layer_norm_backward(dy, x, w, mean, rstd)
        for over_x in (False, True):
            d, v = dy.clone(), x.clone()
            out = v if over_x else d
            got = amq.layer_norm_backward(d, v, w, mean, rstd, out=out)
            assert got[0] is out
            for name, p, q in zip(("dx", "dweight", "dbias"), got, apart):
                assert torch.equal(p, q), (rows, name, "over x" if over_x else "over dy")


@pytest.mark.parametrize("rows,n", [(1, 3), (257, 3), (1000, 2), (70000, 5), (300, 7), (4, 17000), (2100, 16385)])
@pytest.mark.parametrize("dtype", DTYPES)
def test_against_the_formulas(amq, rows, n, dtype):
    x, w, b = case(rows + n, rows, n, dtype, torch.float32)
    check_forward(amq.layer_norm(x.to(DEV), w.to(DEV), b.to(DEV), 1e-5), x, w, b, 1e-5, dtype, "%dx%d" % (rows, n))
    check_backward(amq, rows, n, dtype, torch.float32)


@pytest.mark.parametrize("n,dtype", [(3, torch.float32), (7, torch.bfloat16)])
def test_more_short_rows_than_a_grid_has_workgroups(amq, n, dtype):
    """Forward and backward against the formulas in binary64, on the card."""
    rows = (1 << 22) + 5
    g = torch.Generator(device=DEV).manual_seed(1)
    x = (torch.randn(rows, n, generator=g, device=DEV) + 0.5).to(dtype)
    dy = torch.randn(rows, n, generator=g, device=DEV).to(dtype)
    w, b = 1 + 0.2 * torch.randn(n, generator=g, device=DEV), torch.randn(n, generator=g, device=DEV)
    y, mean, rstd = amq.layer_norm(x, w, b)
    x64, w64 = x.double(), w.double()
    mean64 = x64.mean(1, keepdim=True)
    rstd64 = ((x64 - mean64).square().mean(1, keepdim=True) + 1e-5).rsqrt()
    ref = (x64 - mean64) * rstd64 * w64 + b.double()
    size = 2 * (x64.abs() + x64.abs().mean(1, keepdim=True)) * rstd64 * w64.abs() + b.double().abs() + ref.abs()
    assert bool(((y.double() - ref).abs() <= 96 * U * size + half_ulp(dtype) * ref.abs() + smallest(dtype)).all())
    dx, dw, db = amq.layer_norm_backward(dy, x, w, mean, rstd)
    d, r = dy.double(), rstd.double()[:, None]
    z = (x64 - mean.double()[:, None]) * r
    gz = d * w64
    ref = r * (gz - gz.mean(1, keepdim=True) - z * (gz * z).mean(1, keepdim=True))
    # z is a difference of rounded values; every term of dx is of this size at most
    zs = (x64.abs() + mean.double().abs()[:, None]) * r
    size = r * (gz.abs() + gz.abs().mean(1, keepdim=True) + 2 * zs * (gz.abs() * zs).mean(1, keepdim=True))
    assert bool(((dx.double() - ref).abs() <= 96 * U * size + half_ulp(dtype) * ref.abs() + smallest(dtype)).all())
    # sums over rows: thousands of terms in a row, then as many partial sums
    terms = 96 + rows ** 0.5
    assert bool(((dw.double() - (d * z).sum(0)).abs() <= terms * U * (d.abs() * zs).sum(0)).all())
    assert bool(((db.double() - d.sum(0)).abs() <= terms * U * d.abs().sum(0)).all())
