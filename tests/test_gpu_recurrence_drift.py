"""Units whose gate stays: what a factor 1 - i that is rounded by itself would do to them.

Such a factor is off by up to 2^-25, the same way at every step, so that after T steps a kept state is off by up to T 2^-25 of itself (rms over
gates T 2^-25 / sqrt(3)).  The recurrence keeps h - i h, whose rounding depends on h.  While a state or a map moves by little, consecutive
roundings are alike, so part of that error stays: in binary32 on the CPU, with maps of 16 steps (tiles in workgroups of their own), half of it,
and with maps of 8 steps 0.7.  The fractions asked for here lie between those and 1, which a rounded factor has."""
import numpy as np
import pytest
import torch

from train_util import DEV

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T,n,fraction", [(20000, 512, 0.75), (3000, 16384, 0.85)])
def test_units_that_hold(T, n, fraction):
    import paper_1802_00150_amd as amq
    gate = np.linspace(9.5, 10.5, n).astype(np.float32)
    i = 1 / (1 + np.exp(gate.astype(np.float64)))
    exact = np.exp(T * np.log1p(-i))
    f, h = (1 - i).astype(np.float32), np.ones(n, np.float32)
    for _ in range(T):
        h = f * h
    rounded = float(np.sqrt(np.square(h / exact - 1).mean()))
    assert 0.9 < rounded / (T * 2.0 ** -25 / 3 ** 0.5) < 1.2
    g = torch.from_numpy(gate).to(DEV).expand(T, 1, n).contiguous()
    last = amq.linear_recurrence(g, torch.zeros_like(g), torch.ones(1, n, device=DEV))[1]
    got = float(np.sqrt(np.square(last[0].cpu().numpy() / exact - 1).mean()))
    print("rms of the relative error: %.3g, of a rounded factor %.3g" % (got, rounded))
    assert got < fraction * rounded
