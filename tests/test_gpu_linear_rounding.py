"""What is rounded between the operands and the results of a linear layer.

got = round(ref + e), and the distance of a value to its nearest number of a type changes by no more than the value does, so
|got - ref| <= |round(ref) - ref| + 2 |e| in the 2-norm: e is what is left of everything but the rounding of the result.
"""
import pytest
import torch

from train_util import DEV, U, slope64
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
