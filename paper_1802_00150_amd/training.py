"""Quantization-aware training of a residual block on top of a recurrent layer's hidden states (Sec. 4, "Training":
the forward pass uses the quantized weights, the gradient passes straight through to the full-precision ones, which
are clipped to [-1, 1]).

    normed = layer_norm(h);  y = h + W2_hat gelu(W1_hat normed + b1) + b2,   W_hat = fake_quantize(W)

`layer_norm` and `linear` are the package's operators with their gradients for torch's autograd; `ResidualBlock.step`
runs forward, backward and the update: momentum, orthogonalized matrices, plain steps for vectors, clip.

    python -m paper_1802_00150_amd.training          # a small run that prints its loss
"""
import torch
from torch.autograd.function import once_differentiable

from . import binding


class _LayerNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, eps):
        y, mean, rstd = binding.layer_norm(x.detach(), weight, bias, eps)
        ctx.save_for_backward(x, weight, bias, mean, rstd)
        return y

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        x, weight, bias, mean, rstd = ctx.saved_tensors
        params = ctx.needs_input_grad[1] or ctx.needs_input_grad[2]
        dx, dw, db = binding.layer_norm_backward(dy.contiguous(), x, weight, mean, rstd, params,
                                                 param_dtype=bias.dtype if weight is None and params else None)
        return dx, dw if ctx.needs_input_grad[1] else None, db if ctx.needs_input_grad[2] else None, None


def layer_norm(x, weight=None, bias=None, eps=1e-5):
    """binding.layer_norm's y, differentiable in x, weight and bias."""
    return _LayerNorm.apply(x, weight, bias, eps)


class _Linear(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, W, bias, activation, residual):
        pre = None
        if activation not in (None, "none") and any(ctx.needs_input_grad[:3]):
            pre = torch.empty(*x.shape[:-1], W.shape[0], dtype=x.dtype, device=x.device)
        ctx.activation = activation
        ctx.save_for_backward(x, W, pre)
        return binding.linear(x, W, bias, activation, residual, pre=pre)

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        x, W, pre = ctx.saved_tensors
        need = ctx.needs_input_grad
        dx = dW = db = None
        if any(need[:3]):
            dx, dW, db = binding.linear_backward(dy.contiguous(), x, W, pre, ctx.activation, need[0], need[1], need[2])
        return dx, dW, db, None, dy if need[4] else None


def linear(x, W, bias=None, activation=None, residual=None):
    """binding.linear, differentiable in x, W, bias and residual."""
    return _Linear.apply(x, W, bias, activation, residual)


class ResidualBlock:
    """y = h + W2_hat gelu(W1_hat layer_norm(h) + b1) + b2 with k-bit weights; parameters and momenta in float32."""

    def __init__(self, units, inner, k=2, T=2, device="cuda", seed=0, lr=0.02, momentum=0.95):
        g = torch.Generator(device=device).manual_seed(seed)

        def matrix(rows, cols):
            return (torch.randn(rows, cols, generator=g, device=device) * cols ** -0.5).requires_grad_()

        self.k, self.T, self.lr, self.momentum = k, T, lr, momentum
        self.W1, self.W2 = matrix(inner, units), matrix(units, inner)
        self.b1 = torch.zeros(inner, device=device, requires_grad=True)
        self.b2 = torch.zeros(units, device=device, requires_grad=True)
        self.weight = torch.ones(units, device=device, requires_grad=True)
        self.bias = torch.zeros(units, device=device, requires_grad=True)
        self.matrices, self.vectors = [self.W1, self.W2], [self.b1, self.b2, self.weight, self.bias]
        self.moments = [torch.zeros_like(p) for p in self.matrices + self.vectors]

    def forward(self, h):
        """h [..., units] in float32, bfloat16 or float16; the products run in its type."""
        W1, W2 = (binding.fake_quantize(W, self.k, self.T).to(h.dtype) for W in self.matrices)
        normed = layer_norm(h, self.weight, self.bias)
        inner = linear(normed, W1, self.b1.to(h.dtype), "gelu")
        return linear(inner, W2, self.b2.to(h.dtype), residual=h)

    def step(self, h, loss):
        """One step on `loss` (a function of the block's output); returns its value."""
        value = loss(self.forward(h))
        params = self.matrices + self.vectors
        grads = torch.autograd.grad(value, params)
        with torch.no_grad():
            for p, g, m in zip(params, grads, self.moments):
                m.mul_(self.momentum).add_(g)
                if p.dim() == 2:
                    # the update's singular values are near 1: its size follows the matrix's, not the gradient's
                    p.add_(binding.orthogonalize(m), alpha=-self.lr * max(1.0, p.shape[0] / p.shape[1]) ** 0.5)
                    binding.clip_(p)
                else:
                    p.sub_(m, alpha=self.lr)
        return value.detach()


def main():
    units, rows = 300, 35 * 20
    g = torch.Generator(device="cuda").manual_seed(1)
    h = torch.tanh(torch.randn(rows, units, generator=g, device="cuda"))
    target = h + torch.tanh(h @ torch.randn(units, units, generator=g, device="cuda") * units ** -0.5)
    block = ResidualBlock(units, 4 * units)
    for i in range(50):
        value = block.step(h, lambda y: (y - target).square().mean())
        if i % 10 == 0 or i == 49:
            print("step %d: mean squared error %.5f" % (i, value.item()), flush=True)


if __name__ == "__main__":
    main()
