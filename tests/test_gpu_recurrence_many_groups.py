"""Recurrences whose workgroups have 2^32 threads and more together, which one launch cannot have: a padded batch whose entries all have their full
length is the same batch without lengths, whose channels fill the lanes of a wave and take a 64th of the workgroups."""
import pytest
import torch

from train_util import DEV

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def amq():
    import paper_1802_00150_amd as amq
    return amq


def normal(seed, shape, dtype):
    return torch.empty(shape, dtype=dtype, device=DEV).normal_(generator=torch.Generator(device=DEV).manual_seed(seed))


@pytest.mark.parametrize("T,B", [(128, 1 << 22), (1 << 20, 1 << 10)])
def test_forward(amq, T, B):
    """One tile of 16 waves for each of 2^22 entries; 4096 tiles in workgroups of their own for each of 1024."""
    gate, x = (normal(i, (T, B, 1), torch.bfloat16) for i in (1, 2))
    lengths = torch.full((B,), T, dtype=torch.int64, device=DEV)
    want = amq.linear_recurrence(gate, x)
    got = amq.linear_recurrence(gate, x, lengths=lengths)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    assert bool((got[1] != 0).all())


def test_backward(amq):
    """4096 tiles in workgroups of their own for each of 1024 entries."""
    T, B = 1 << 19, 1 << 10
    gate, x, dhs = (normal(i, (T, B, 1), torch.float32) for i in (1, 2, 3))
    lengths = torch.full((B,), T, dtype=torch.int64, device=DEV)
    h0 = torch.zeros(B, 1, device=DEV)
    states = amq.linear_recurrence(gate, x, h0, states=True)[2]
    want = amq.linear_recurrence_backward(dhs, gate, x, h0, states)
    got = amq.linear_recurrence_backward(dhs, gate, x, h0, states, lengths=lengths)
    assert all(torch.equal(p, q) for p, q in zip(got, want))
    assert bool((got[2] != 0).all())
