"""Gradients of layer norm's parameters come with the digits of the parameter."""
import pytest
import torch

from train_util import DEV, U, assert_within, rand

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_bias_without_a_weight(dtype):
    """A float32 bias keeps a float32 gradient where there is no weight: sums of `rows` terms of binary32 and no other rounding."""
    from paper_1802_00150_amd import training
    rows, n = 300, 65
    x, c = rand(5, rows, n).to(dtype).to(DEV), rand(6, rows, n).to(dtype)
    bias = rand(7, n).to(DEV).requires_grad_()
    training.layer_norm(x, None, bias).backward(c.to(DEV))
    assert bias.grad.dtype == torch.float32
    assert_within(bias.grad, c.double().sum(0), (96 + rows) * U * c.double().abs().sum(0), "dbias")


def test_the_type_is_the_caller_s_where_there_is_no_weight():
    import paper_1802_00150_amd as amq
    x = rand(8, 30, 50).to(torch.bfloat16).to(DEV)
    dy, w = rand(9, 30, 50).to(torch.bfloat16).to(DEV), torch.ones(50, dtype=torch.bfloat16, device=DEV)
    _, mean, rstd = amq.layer_norm(x)
    plain, wide = (amq.layer_norm_backward(dy, x, None, mean, rstd, param_dtype=t) for t in (None, torch.float32))
    assert torch.equal(plain[0], wide[0])
    for p, q in zip(plain[1:], wide[1:]):
        assert p.dtype == torch.bfloat16 and q.dtype == torch.float32 and torch.equal(p, q.to(torch.bfloat16))
    for weight, dtype in ((w, torch.float32), (None, torch.float16), (None, torch.float64)):
        with pytest.raises((amq.AmqError, ValueError)):
            amq.layer_norm_backward(dy, x, weight, mean, rstd, param_dtype=dtype)
