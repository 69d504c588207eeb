"""Products whose results fill the card with tiles of 192 and 256, in the three orders of their operands, against the formulas
in binary64 (computed on the card: library products of binary64).

Tolerances are those of the smaller products, per element: (terms + 16) U of the sum of magnitudes, a rounding of the result.
"""
import pytest
import torch

from train_util import DEV, U, half_ulp, rand, smallest

pytestmark = pytest.mark.gpu
HALVES = [torch.bfloat16, torch.float16]


@pytest.fixture(scope="module")
def amq():
    import paper_1802_00150_amd as amq
    return amq


def operand(seed, rows, cols, dtype, scale=1.0):
    return rand(seed, rows, cols, scale=scale).to(dtype).to(DEV)


def check(got, a, b, dtype, terms, bias=None):
    """got = a b (binary64) + bias; float operands are split into 22 bits"""
    ref, size = a @ b, a.abs() @ b.abs()
    if bias is not None:
        ref, size = ref + bias, size + bias.abs()
    tol = ((terms + 16) * U + (2.0 ** -21 if dtype == torch.float32 else 0.0)) * size + half_ulp(dtype) * ref.abs() * 1.01 + smallest(dtype)
    assert got.dtype == dtype and got.shape == ref.shape
    assert bool(((got.double() - ref).abs() <= tol).all())  # (NaN counts as off)


# result M x N over k: 16 x 16 tiles of 192 with ragged ends, 16 x 16 of 256; k a multiple of neither 64 nor 8 too
@pytest.mark.parametrize("M,N,k", [(3000, 3050, 1000), (3010, 2960, 1001), (4000, 4090, 600), (4096, 3900, 333)])
@pytest.mark.parametrize("dtype", HALVES)
def test_every_order_of_operands(amq, M, N, k, dtype):
    x, W, bias = operand(1, M, k, dtype), operand(2, N, k, dtype, k ** -0.5), operand(3, 1, N, dtype)[0]
    check(amq.linear(x, W, bias), x.double(), W.double().t().contiguous(), dtype, k, bias.double())
    # dx = dy W: M x N over k features out
    dy, W = operand(4, M, k, dtype), operand(5, k, N, dtype, k ** -0.5)
    x = operand(6, M, N, dtype)
    dx, dW, db = amq.linear_backward(dy, x, W, None, None, True, False, False)
    assert dW is None and db is None
    check(dx, dy.double(), W.double(), dtype, k)
    # dW = dy^T x: M x N over k rows
    dy, x = operand(7, k, M, dtype, k ** -0.5), operand(8, k, N, dtype)
    W = operand(9, M, N, dtype)
    dx, dW, db = amq.linear_backward(dy, x, W, None, None, False, True, False)
    assert dx is None and db is None
    check(dW, dy.double().t().contiguous(), x.double(), dtype, k)


# both gradients in one launch or in two, with tiles of 64 and 128, the longer contraction in either of them
@pytest.mark.parametrize("rows,k,n", [(2000, 2200, 1700), (1700, 2200, 2010), (3300, 2250, 700), (700, 2250, 3300), (2390, 3990, 320), (330, 3810, 380), (1130, 3920, 480),
                                      (430, 3810, 390), (8960, 300, 310), (300, 1500, 8000)])
@pytest.mark.parametrize("dtype", [torch.float32] + HALVES)
def test_both_gradients(amq, rows, k, n, dtype):
    dy, x, W = operand(1, rows, n, dtype), operand(2, rows, k, dtype), operand(3, n, k, dtype, n ** -0.5)
    dx, dW, db = amq.linear_backward(dy, x, W)
    check(dx, dy.double(), W.double(), dtype, n)
    check(dW, dy.double().t().contiguous(), x.double(), dtype, rows)
    check(db[None], torch.ones(1, rows, dtype=torch.float64, device=DEV), dy.double(), dtype, rows)


@pytest.mark.parametrize("rows,cols", [(3900, 4200), (4200, 3900), (5500, 5610)])
def test_orthogonalized_updates(amq, rows, cols):
    """Two steps: the symmetric products' lower tiles, the update, and the last one's result."""
    a, b, c = 3.4445, -4.7750, 2.0315
    G = rand(rows, rows, cols).to(torch.bfloat16).to(DEV)
    got = amq.orthogonalize(G, steps=2)
    X = G.double() if rows <= cols else G.double().t().contiguous()
    X = X / X.norm()
    for _ in range(2):
        A = X @ X.t().contiguous()
        X = a * X + (b * A + c * (A @ A)) @ X
    ref = X if rows <= cols else X.t()
    # iterates of 11 bits: 1.5e-3 over five steps, beside the rounding of the result
    assert float((got.double() - ref).norm() / ref.norm()) <= 1.5e-3 + half_ulp(torch.bfloat16)
    assert float((got.double() - ref).abs().max()) <= 0.02 * float(ref.abs().max())


@pytest.mark.parametrize("dtype", [torch.float32] + HALVES)
def test_offsets_past_32_bits(amq, dtype):
    """Rows 2^22 entries apart, the last ones beyond 2^32 entries: the results are those of the same rows side by side."""
    rows, k, n, apart = 1100, 304, 208, 1 << 22

    def spread(t, first):
        wide = torch.empty(rows, apart, dtype=dtype, device=DEV)[:, first:first + t.shape[1]]
        return wide.copy_(t)

    x, dy, W, bias = operand(1, rows, k, dtype), operand(2, rows, n, dtype), operand(3, n, k, dtype, k ** -0.5), operand(4, 1, n, dtype)[0]
    far_x, far_dy = spread(x, 8), spread(dy, apart - n)
    assert torch.equal(amq.linear(far_x, W, bias, "relu", far_dy, out=far_dy), amq.linear(x, W, bias, "relu", dy))
    far_dy.copy_(dy)
    pre = amq.linear(x, W)
    far_pre = spread(pre, 16)
    for got, ref in zip(amq.linear_backward(far_dy, far_x, W, far_pre, "tanh") + amq.linear_backward(far_dy, far_x, W),
                        amq.linear_backward(dy, x, W, pre, "tanh") + amq.linear_backward(dy, x, W)):
        assert torch.equal(got, ref)
    assert torch.equal(amq.orthogonalize(far_x, out=spread(x, 0)), amq.orthogonalize(x))
    y, mean, rstd = amq.layer_norm(x)
    far_y, far_mean, far_rstd = amq.layer_norm(far_x, out=spread(x, 0))
    assert torch.equal(far_y, y) and torch.equal(far_mean, mean) and torch.equal(far_rstd, rstd)
    g = operand(5, rows, k, dtype)
    for got, ref in zip(amq.layer_norm_backward(spread(g, 8), far_x, None, mean, rstd), amq.layer_norm_backward(g, x, None, mean, rstd)):
        assert torch.equal(got, ref)
    del far_x, far_dy, far_pre, far_y
    torch.cuda.empty_cache()
