"""Results that the caller gives, beside autograd: a graph that saved what they held says so, and those that require a gradient are refused."""
import pytest
import torch

from train_util import DEV, rand

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def amq():
    import paper_1802_00150_amd as amq
    return amq


@pytest.fixture(scope="module")
def training():
    from paper_1802_00150_amd import training
    return training


T, B, N = 20, 3, 48


def sequence(seed):
    return rand(seed, T, B, N).to(DEV)


def test_a_saved_state_that_a_later_call_overwrites(amq, training):
    """The state in front of a sequence is saved for its backward pass."""
    gate, x, state = sequence(1).requires_grad_(), sequence(2), rand(3, B, N).to(DEV)
    want = torch.autograd.grad(training.linear_recurrence(gate, x, state.clone())[0].sum(), gate)[0]
    hs, _ = training.linear_recurrence(gate, x, state)
    amq.linear_recurrence(sequence(4), sequence(5), state, h_out=state)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        torch.autograd.grad(hs.sum(), gate)
    hs, _ = training.linear_recurrence(gate, x, state)
    amq.linear_recurrence(sequence(4), sequence(5), state)
    assert torch.autograd.grad(hs.sum(), gate)[0].shape == want.shape


def saved(training, value):
    """A graph that has saved `value` (a product keeps the other factor)."""
    one = torch.ones_like(value).requires_grad_()
    return one, (one * value).sum()


def overwrites(amq):
    """Calls that write a tensor of the caller's, and those tensors."""
    g, x, d, a, r = sequence(1), sequence(2), sequence(3), rand(4, 30, N).to(DEV), rand(5, 30, N).to(DEV)
    W, v = rand(6, N, N).to(DEV), rand(7, N).to(DEV)
    new = torch.empty_like
    hs, h, dg, dx, y, n, o, z, p, m, t, u, e = new(x), new(x[0]), new(x), new(x), r.clone(), new(a), new(W), new(a), new(a), new(a), v.clone(), new(v), new(a)
    mean, rstd = amq.layer_norm(a)[1:]
    yield lambda: amq.linear_recurrence(g, x, out=hs, h_out=h), (hs, h)
    yield lambda: amq.linear_recurrence_backward(d, g, x, dgate=dg, dx=dx), (dg, dx)
    yield lambda: amq.block_norm(a, y, out=y, out_normed=n), (y, n)
    yield lambda: amq.clip_gradients([t], 0.5), (t,)
    yield lambda: amq.clip_gradients([v], 0.5, out=[u]), (u,)
    yield lambda: amq.orthogonalize(W, out=o), (o,)
    yield lambda: amq.linear(a, W, activation="relu", out=z, pre=p), (z, p)
    yield lambda: amq.layer_norm(a, out=m), (m,)
    yield lambda: amq.layer_norm_backward(a, a, None, mean, rstd, out=e), (e,)


def test_every_given_result_counts_as_written(amq, training):
    for i, (call, results) in enumerate(overwrites(amq)):
        graphs = [saved(training, r) for r in results]
        before = [r._version for r in results]
        call()
        assert all(r._version > v for r, v in zip(results, before)), i
        for one, value in graphs:
            with pytest.raises(RuntimeError, match="modified by an inplace operation"):
                torch.autograd.grad(value, one)


def test_operands_and_own_results_do_not(amq):
    g, x, h = sequence(1), sequence(2), rand(3, B, N).to(DEV)
    hs, last, _ = amq.linear_recurrence(g, x, h)
    assert [t._version for t in (g, x, h, hs, last)] == [0] * 5
    amq.gradient_norm([g, x])
    assert g._version == x._version == 0


def test_inference_tensors(amq):
    """They have no version."""
    with torch.inference_mode():
        g, x, h = sequence(1), sequence(2), rand(3, B, N).to(DEV)
        want = amq.linear_recurrence(g, x, h)[1]
        assert amq.linear_recurrence(g, x, h, h_out=h)[1] is h and torch.equal(h, want)
        amq.clip_gradients([x], 0.1)


def test_results_that_require_a_gradient(amq):
    g, x, d, a, r = sequence(1), sequence(2), sequence(3), rand(4, 30, N).to(DEV), rand(5, 30, N).to(DEV)
    leaf = lambda t: torch.empty_like(t).requires_grad_()  # noqa: E731
    for name, call in (("linear_recurrence", lambda: amq.linear_recurrence(g, x, out=leaf(x))), ("linear_recurrence", lambda: amq.linear_recurrence(g, x, h_out=leaf(x[0]))),
                       ("linear_recurrence_backward", lambda: amq.linear_recurrence_backward(d, g, x, dgate=leaf(x))),
                       ("linear_recurrence_backward", lambda: amq.linear_recurrence_backward(d, g, x, dx=leaf(x))),
                       ("block_norm", lambda: amq.block_norm(a, r, out=leaf(r))), ("block_norm", lambda: amq.block_norm(a, r, out_normed=leaf(a))),
                       ("clip_gradients", lambda: amq.clip_gradients([a], 1.0, out=[leaf(a)]))):
        with pytest.raises(amq.AmqError, match=name):
            call()
        with torch.no_grad():
            call()


def test_a_refused_call_writes_nothing(amq):
    """... and counts as having written nothing."""
    g, x = sequence(1), sequence(2)
    out = torch.empty_like(x)
    with pytest.raises(amq.AmqError):
        amq.linear_recurrence(g, x, out=out, h_out=out[0])
    assert out._version == 0
