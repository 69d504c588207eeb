"""What is rounded between the operands and the results of a linear layer.

got = round(ref + e), and the distance of a value to its nearest number of a type changes by no more than the value does, so
|got - ref| <= |round(ref) - ref| + 2 |e| in the 2-norm: e is what is left of everything but the rounding of the result.
"""
import pytest
import torch

from train_util import DEV, U, assert_within, rand, slope64
from test_gpu_linear import inputs

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def amq():
    import paper_1802_00150_amd as amq
    return amq


# d read by one product or two launched together, tiles of 32 to 256, split contractions, sizes that are no multiple of anything
@pytest.mark.parametrize("rows,k,n", [(70, 80, 90), (300, 1000, 66), (64, 2048, 64), (700, 650, 130), (2300, 200, 1800), (3600, 1030, 1100), (4100, 72, 72)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("act", ["gelu", "silu", "sigmoid", "tanh", "relu"])
def test_the_gradient_between_slope_and_products(amq, rows, k, n, dtype, act):
    """d = dy act'(pre) reaches both products with 16 bits or more: its two parts leave 2^-16 of it, independent from entry to entry; slopes
    err by 8 U (1 + z^2), sums of binary32 by less than 2^-20."""
    x, W, _, dy = inputs(rows + k + n, rows, k, n, dtype)
    x, W, dy = x.to(DEV), W.to(DEV), (dy.float() / rows).to(dtype).to(DEV)
    pre = (x.double() @ W.double().t().contiguous()).to(dtype)
    dx, dW, db = amq.linear_backward(dy, x, W, pre, act)
    d = dy.double() * slope64(pre.double(), act)
    x64, W64, dt = x.double(), W.double(), d.t().contiguous()
    share = 2.0 ** -16 + 2.0 ** -20 + 8 * U * 16
    for got, ref, terms, what in ((dx, d @ W64, (d * d) @ (W64 * W64), "dx"), (dW, dt @ x64, (dt * dt) @ (x64 * x64), "dW")):
        rounding = float((ref.to(dtype).double() - ref).norm())
        e = share * float(terms.sum().sqrt())
        assert float((got.double() - ref).norm()) <= rounding + 2 * e, (what, float((got.double() - ref).norm()), rounding, e)
    assert float((db.double() - d.sum(0)).norm()) <= float((d.sum(0).to(dtype).double() - d.sum(0)).norm()) + 2 * share * float((d * d).sum().sqrt())


# each gradient in a launch of its own, where tiles of 64, 128, 192 and 256 and splits of either contraction are taken; k, n and rows odd, and multiples
# of 8 that are read in place
@pytest.mark.parametrize("rows,k,n", [(9000, 72, 200), (20001, 40, 47), (1500, 300, 8000), (3000, 1000, 3050), (3000, 3050, 500), (500, 3050, 3000), (8960, 2050, 1024),
                                      (8960, 4096, 200), (1024, 4096, 8960)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_each_gradient_alone(amq, rows, k, n, dtype):
    """The same bound for the product of either gradient by itself."""
    x, W, _, dy = inputs(rows + k + n, rows, k, n, dtype)
    x, W, dy = x.to(DEV), W.to(DEV), (dy.float() / rows).to(dtype).to(DEV)
    pre = amq.linear(x, W)
    d = dy.double() * slope64(pre.double(), "gelu")
    dx, none, none2 = amq.linear_backward(dy, x, W, pre, "gelu", True, False, False)
    assert none is None and none2 is None
    dW = amq.linear_backward(dy, x, W, pre, "gelu", False, True, False)[1]
    share = 2.0 ** -16 + 2.0 ** -20 + 8 * U * 16
    for got, a, b, what in ((dx, d, W.double(), "dx"), (dW, d.t().contiguous(), x.double(), "dW")):
        ref = a @ b
        e, rounding = share * float(((a * a) @ (b * b)).sum().sqrt()), float((ref.to(dtype).double() - ref).norm())
        assert float((got.double() - ref).norm()) <= rounding + 2 * e, (what, float((got.double() - ref).norm()), rounding, e)
        assert float((got.double() - ref).abs().max()) <= 0.02 * float(ref.abs().max()), what


@pytest.mark.parametrize("rows", [9, 40, 300])
@pytest.mark.parametrize("far", [10, 18, 24, 28])
def test_float_entries_far_below_the_largest_of_their_row(amq, rows, far):
    """Entries 2^-far of their row's largest, whose own products are all that a result has (W is 0 at the large ones).  An entry of a split
    operand is off by 2^-23 of itself or 2^-39 of its row's largest; the product of two low parts, 2^-22, is left out."""
    k, n = 200, 72
    x, W = rand(far, rows, k), rand(far + 1, n, k)
    x[:, ::2] *= 2.0 ** -far
    W[:, 1::2] = 0

    def off(t):
        return torch.maximum(2.0 ** -23 * t.abs(), 2.0 ** -39 * t.abs().amax(1, keepdim=True)) * (t != 0)

    ref, a, w = x.double() @ W.double().t(), x.double().abs(), W.double().abs()
    tol = ((k + 16) * U + 2.0 ** -22) * (a @ w.t()) + off(x.double()) @ w.t() + a @ off(W.double()).t() + off(x.double()) @ off(W.double()).t()
    assert_within(amq.linear(x.to(DEV), W.to(DEV)), ref, tol + U * ref.abs(), "y")
