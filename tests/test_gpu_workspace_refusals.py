"""Workspaces that a kernel could not write."""
import pytest
import torch

from train_util import DEV, rand

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def amq():
    import paper_1802_00150_amd as amq
    return amq


def test_workspaces_elsewhere_or_apart(amq):
    T, n = 5000, 64
    g, x, d = (rand(i, T, 1, n).to(DEV) for i in (1, 2, 3))
    a, W, w = rand(4, 300, n).to(DEV), rand(5, n, n).to(DEV), rand(6, n).to(DEV)
    states = amq.linear_recurrence(g, x, states=True)[2]
    y, _, stats = amq.block_norm(a, a.clone(), w)
    calls = {
        "recurrence": lambda ws: amq.linear_recurrence(g, x, ws=ws),
        "its gradient": lambda ws: amq.linear_recurrence_backward(d, g, x, None, states, ws=ws),
        "join's gradient": lambda ws: amq.block_norm_backward(a, a, a, y, stats, w, ws=ws),
        "clipping": lambda ws: amq.clip_gradients([a], 1e9, ws=ws),
        "norm": lambda ws: amq.gradient_norm([a], ws=ws),
        "linear": lambda ws: amq.linear(a, W, ws=ws),
        "updates": lambda ws: amq.orthogonalize(W, ws=ws),
    }
    large = 1 << 24
    assert large >= amq.linear_recurrence_workspace(T, 1, n, x.dtype, DEV).numel() > 0
    for name, call in calls.items():
        with pytest.raises(amq.AmqError, match="workspace"):
            call(torch.empty(large, dtype=torch.uint8))
        # as many entries as a workspace has bytes, in a few bytes of memory
        with pytest.raises(ValueError, match="workspace"):
            call(torch.empty(1, dtype=torch.uint8, device=DEV).expand(large))
        call(torch.empty(large, dtype=torch.uint8, device=DEV))
