"""Layer normalization of rows outside the range whose entries a wave or workgroup holds: of more than 16384 entries, and of less than 16 bytes.
"""
import pytest
import torch

from train_util import DEV, DTYPES, rand
from test_gpu_layer_norm import case

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def amq():
    import paper_1802_00150_amd as amq
    return amq


# (the forms for 16 bytes and more beside them: with four waves per row, with one, with sixteen)
@pytest.mark.parametrize("n", [3, 7, 8, 301, 1500, 16384, 16385, 20011])
@pytest.mark.parametrize("dtype", DTYPES)
def test_backward_in_place(amq, n, dtype):
    """dx over dy or over x: all three gradients are those of a dx of its own."""
    for rows in (5, 70, 300):
        x, w, _ = case(rows + n, rows, n, dtype, torch.float32)
        x, w, dy = x.to(DEV), w.to(DEV), rand(1, rows, n).to(dtype).to(DEV)
        _, mean, rstd = amq.layer_norm(x)
        apart = amq.layer_norm_backward(dy, x, w, mean, rstd)
        for over_x in (False, True):
            d, v = dy.clone(), x.clone()
            out = v if over_x else d
            got = amq.layer_norm_backward(d, v, w, mean, rstd, out=out)
            assert got[0] is out
            for name, p, q in zip(("dx", "dweight", "dbias"), got, apart):
                assert torch.equal(p, q), (rows, name, "over x" if over_x else "over dy")
