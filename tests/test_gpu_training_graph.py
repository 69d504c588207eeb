"""Operators that record no graph say so instead of returning a result without one."""
import pytest
import torch

from train_util import DEV, rand

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def amq():
    import paper_1802_00150_amd as amq
    return amq


def test_no_gradient_is_dropped(amq):
    x, W, b, r = rand(1, 20, 16).to(DEV), rand(2, 16, 16).to(DEV), rand(3, 16).to(DEV), rand(4, 20, 16).to(DEV)
    calls = {"linear": (amq.linear, (x, W, b, None, r), (0, 1, 2, 4)), "layer_norm": (amq.layer_norm, (x, b, b.clone()), (0, 1, 2)),
             "orthogonalize": (amq.orthogonalize, (W,), (0,))}
    for name, (f, args, operands) in calls.items():
        plain = f(*args)
        for i in operands:
            with_grad = list(args)
            with_grad[i] = args[i].clone().requires_grad_()
            with pytest.raises(amq.AmqError, match=name):
                f(*with_grad)
            with torch.no_grad():
                got = f(*with_grad)
            for p, q in zip(got if isinstance(got, tuple) else (got,), plain if isinstance(plain, tuple) else (plain,)):
                assert torch.equal(p, q) and not p.requires_grad
    with pytest.raises(amq.AmqError, match="linear"):
        amq.linear(x, amq.fake_quantize(W.clone().requires_grad_(), 2))


def test_backward_calls_take_parameters(amq):
    """Gradients are asked for with the parameters themselves at hand."""
    x, W, dy = rand(1, 20, 16).to(DEV), rand(2, 12, 16).to(DEV).requires_grad_(), rand(3, 20, 12).to(DEV)
    assert torch.equal(amq.linear_backward(dy, x, W)[0], amq.linear_backward(dy, x, W.detach())[0])
