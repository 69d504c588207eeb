"""Helpers for the tests of the training operators: inputs, and the plain forms in binary64 on the CPU."""
import math

import torch

DEV = "cuda:0"
DTYPES = [torch.float32, torch.bfloat16, torch.float16]
U = 2.0 ** -24  # unit roundoff of binary32
ACTS = ["none", "relu", "gelu", "silu", "sigmoid", "tanh"]


def half_ulp(dtype):
    """Largest relative error of one rounding to dtype."""
    return torch.finfo(dtype).eps / 2


def smallest(dtype):
    """Half of the smallest step of dtype: the error of a rounding near 0."""
    return {torch.float32: 0.0, torch.bfloat16: 0.0, torch.float16: 2.0 ** -25}[dtype]


def rand(seed, *shape, scale=1.0, dtype=torch.float32):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(*shape, generator=g) * scale).to(dtype)


def act64(z, name):
    if name == "relu":
        return torch.where(z > 0, z, torch.zeros_like(z))
    if name == "gelu":
        return 0.5 * z * (1 + torch.erf(z / math.sqrt(2.0)))
    if name == "silu":
        return z / (1 + torch.exp(-z))
    if name == "sigmoid":
        return 1 / (1 + torch.exp(-z))
    if name == "tanh":
        return torch.tanh(z)
    return z


def slope64(z, name):
    if name == "relu":
        return (z > 0).double()
    if name == "gelu":
        return 0.5 * (1 + torch.erf(z / math.sqrt(2.0))) + z * torch.exp(-0.5 * z * z) / math.sqrt(2 * math.pi)
    s = 1 / (1 + torch.exp(-z))
    if name == "silu":
        return s * (1 + z * (1 - s))
    if name == "sigmoid":
        return s * (1 - s)
    if name == "tanh":
        return 1 - torch.tanh(z) ** 2
    return torch.ones_like(z)


def assert_within(got, ref, tol, what):
    got, ref = got.detach().cpu().double(), ref.double()
    assert got.shape == ref.shape, (what, got.shape, ref.shape)
    bad = ~((got - ref).abs() <= tol)  # (NaN counts)
    assert not bad.any(), "%s: %d of %d off, worst %g at a tolerance of %g" % (
        what, int(bad.sum()), bad.numel(), float((got - ref).abs().max()), float((tol if torch.is_tensor(tol) else torch.tensor(tol)).max()))


def relative(got, ref):
    """2-norm of the difference over the 2-norm of the reference."""
    ref = ref.double()
    n = float(ref.norm())
    return float((got.detach().cpu().double() - ref).norm()) / n if n else float(got.detach().cpu().double().norm())
