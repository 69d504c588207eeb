"""Orthogonalized updates of matrices whose norm's reciprocal binary32 does not hold, without eps."""
import pytest
import torch

from train_util import DEV, DTYPES, relative
from test_gpu_orthogonalize import COEF, gradient, ortho64

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def amq():
    import paper_1802_00150_amd as amq
    return amq


@pytest.mark.parametrize("dtype", DTYPES[:2])
@pytest.mark.parametrize("steps", [0, 5])
def test_small_norms_without_eps(amq, dtype, steps):
    """Norms whose reciprocal leaves binary32, alone or times the iterates' scale.  (Reference from the same, possibly subnormal, values.)"""
    for scale in (1e-33, 1e-35, 1e-37, 1e-38):
        G = (gradient(3, 90, 140) * scale).to(dtype)
        ref = ortho64(G, steps, COEF, 0.0)
        rounding = 0.0 if dtype == torch.float32 else relative(ref.to(dtype), ref)
        assert relative(amq.orthogonalize(G.to(DEV), steps=steps, eps=0.0), ref) <= rounding + 2e-5, scale
