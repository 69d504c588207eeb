"""Orthogonalized updates of bfloat16 matrices: the result is off by the rounding of the result alone.

got = round(ref + e), and the distance of a value to its nearest bfloat16 changes by no more than the value does, so
|got - ref| <= |round(ref) - ref| + 2 |e| in the 2-norm.  e is what 22-bit iterates leave, 1e-5 of the result (the bound that float
matrices are held to).
"""
import pytest
import torch

from train_util import DEV, DTYPES, relative
from test_gpu_orthogonalize import gradient, ortho64

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def amq():
    import paper_1802_00150_amd as amq
    return amq


# wide, square and tall; the smaller size on either side of 512, and sizes that are no multiple of anything
@pytest.mark.parametrize("rows,cols", [(64, 64), (511, 700), (512, 512), (513, 1300), (1030, 1100), (1500, 520)])
@pytest.mark.parametrize("dtype", DTYPES[1:])
def test_only_the_result_is_rounded(amq, rows, cols, dtype):
    G = gradient(rows + cols, rows, cols).to(dtype)
    got, ref = amq.orthogonalize(G.to(DEV)), ortho64(G)
    rounding = relative(ref.to(dtype), ref)
    assert relative(got, ref) <= rounding + 2e-5, (relative(got, ref), rounding)
