"""A NaN spoils the results that it enters, whatever the activation, and no others."""
import pytest
import torch

from train_util import ACTS, DEV, DTYPES
from test_gpu_linear import inputs

pytestmark = pytest.mark.gpu
NAN = float("nan")


@pytest.fixture(scope="module")
def amq():
    import paper_1802_00150_amd as amq
    return amq


def spoiled_only(got, ref, row=None, col=None):
    m = torch.zeros(got.shape, dtype=torch.bool, device=DEV)
    m[(slice(None) if row is None else row,) + ((slice(None) if col is None else col,) if got.dim() == 2 else ())] = True
    assert torch.equal(got[~m], ref[~m]) and bool(torch.isnan(got[m]).all())


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,k,n", [(5, 70, 33), (150, 90, 130)])
def test_nan(amq, rows, k, n, dtype, act):
    x, W, b, dy = (t.to(DEV) for t in inputs(21, rows, k, n, dtype))

    def with_entry(t, at, v):
        t = t.clone()
        t[at] = v
        return t

    y = [amq.linear(with_entry(x, (3, 7), v), W, b, act) for v in (NAN, 0.0)]
    spoiled_only(*y, row=3)
    y = [amq.linear(x, with_entry(W, (4, 6), v), b, act) for v in (NAN, 0.0)]
    spoiled_only(*y, col=4)
    y = [amq.linear(x, W, with_entry(b, 9, v), act) for v in (NAN, 0.0)]
    spoiled_only(*y, col=9)
    pre = amq.linear(x, W, b)
    for of_pre in (False, True):
        if of_pre and act == "none":
            continue
        # (0 in place of dy's entry: what does not depend on it is the same either way)
        d = [with_entry(dy, (2, 5), 0.0 if of_pre else v) for v in (NAN, 0.0)]
        p = [with_entry(pre, (2, 5), v) if of_pre else pre for v in (NAN, 0.0)]
        got, ref = (amq.linear_backward(a, x, W, c, act) for a, c in zip(d, p))
        spoiled_only(got[0], ref[0], row=2)
        spoiled_only(got[1], ref[1], row=5)
        spoiled_only(got[2], ref[2], row=5)
