"""Captures beside graphs that were recorded outside: refused where torch's backward pass would end the process, and only there."""
import gc

import pytest
import torch

from train_util import DEV, rand

pytestmark = pytest.mark.gpu

T, B, N = 12, 3, 48


@pytest.fixture(scope="module")
def amq():
    import paper_1802_00150_amd as amq
    return amq


@pytest.fixture(scope="module")
def training():
    from paper_1802_00150_amd import training
    return training


def replays(graph, out, again, x):
    """Four replays with other inputs against the same work outside, with synchronizations between."""
    for i in range(4):
        x.copy_(rand(20 + i, *x.shape))
        graph.replay()
        torch.cuda.synchronize()
        want = again()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(out, want)), i


def capture(stream, work):
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        out = work()
    return graph, out


def warm(stream, work):
    with torch.cuda.stream(stream):
        work()
    torch.cuda.synchronize()


def test_without_gradients(training):
    """Serving through the block while a training step's graph is alive: no backward pass can come of it."""
    block = training.RecurrentBlock(N, device=DEV, seed=1)
    h, state = rand(1, T, B, N).to(DEV), rand(2, B, N).to(DEV)
    alive = block.forward(h, state)
    stream = torch.cuda.Stream()

    def serve():
        with torch.no_grad():
            return block.forward(h, state)

    warm(stream, serve)
    graph, out = capture(stream, serve)
    replays(graph, out, serve, h)
    assert alive[0].requires_grad


@pytest.mark.parametrize("name", ["layer_norm", "linear"])
def test_backward_passes_of_the_other_operators(amq, training, name):
    """Their forward pass alone is captured; with its backward pass it is refused, from there, and may be captured once the graph outside is gone."""
    x, W, v = rand(1, 20, N).to(DEV), rand(2, N, N).to(DEV).requires_grad_(), torch.ones(N, device=DEV).requires_grad_()
    w = rand(3, 20, N).to(DEV)
    leaves = [v] if name == "layer_norm" else [W, v]

    def forward():
        return training.layer_norm(x, v) if name == "layer_norm" else training.linear(x, W, v * 1.0, "silu")

    def both():
        y = forward()
        return (y.detach(),) + torch.autograd.grad((y * w).sum(), leaves)

    stream = torch.cuda.Stream()
    alive = forward()
    torch.cuda.synchronize()
    warm(stream, lambda: forward().detach())
    graph, out = capture(stream, lambda: (forward().detach(),))
    replays(graph, out, lambda: (forward().detach(),), x)
    with pytest.raises(amq.AmqError, match=name + ".*still alive"), torch.cuda.graph(torch.cuda.CUDAGraph(), stream=stream):
        both()
    torch.cuda.synchronize()
    # outside of a capture nothing is refused
    assert all(torch.equal(p, q) for p, q in zip(both(), both()))
    del alive
    gc.collect()  # (the exception's frames hold what was recorded)
    warm(stream, both)
    graph, out = capture(stream, both)
    replays(graph, out, both, x)


def accumulator(leaf):
    """What a hook on a leaf's gradient is registered on, and keeps alive."""
    return leaf.view_as(leaf).grad_fn.next_functions[0][0]


def test_hooks_on_leaves(amq, training):
    """One made on the stream that captures is no reason to refuse; one made elsewhere is, for as long as it lives."""
    gate, x, w = rand(1, T, B, N).to(DEV).requires_grad_(), rand(2, T, B, N).to(DEV), rand(3, T, B, N).to(DEV)

    def both():
        hs, _ = training.linear_recurrence(gate, x)
        return (hs.detach(),) + torch.autograd.grad((hs * w).sum(), [gate])

    stream = torch.cuda.Stream()
    hook = accumulator(gate)
    torch.cuda.synchronize()
    with pytest.raises(amq.AmqError, match="hooks"), torch.cuda.graph(torch.cuda.CUDAGraph(), stream=stream):
        both()
    del hook
    gc.collect()
    with torch.cuda.stream(stream):
        hook = accumulator(gate)
        calls = []
        handle = hook.register_hook(lambda *_: calls.append(1))
        both()
    torch.cuda.synchronize()
    graph, out = capture(stream, both)
    replays(graph, out, both, x)
    handle.remove()
