"""Results of the training operators that overlap an operand or another result are refused before any launch (no GPU)."""
import ctypes as C

import pytest

from test_train_refusals import BF16, F32, INVALID, L, NULL, call  # noqa: F401

SIZE = {F32: 4, BF16: 2}


def at(entry, type=F32, base=0x1000000):
    return C.c_void_p(base + entry * SIZE[type])


def apart(i):  # the i-th of many buffers that do not meet
    return C.c_void_p(0x100000000 + i * 0x10000000)


def test_linear(L):
    rows, k, n = 20, 8, 8
    need = L.amq_linear_workspace_bytes(rows, k, n, F32)
    # x at 0 in rows of 8, of 20 where columns of a wider matrix are meant
    args = dict(x=at(0), ld_x=8, W=apart(1), ld_w=8, rows=rows, k=k, n=n, type=F32, bias=apart(2), act=0, residual=apart(3), ld_r=8, y=apart(4), ld_y=8,
                pre=apart(5), ld_pre=8, ws=apart(6), bytes=need, stream=None)
    last = (rows - 1) * 8 + 7
    for bad in (dict(y=at(0)), dict(y=at(last)), dict(y=at(-last)), dict(pre=at(3)), dict(y=at(0), ld_y=9), dict(y=at(-1), ld_y=16),
                dict(ld_x=20, y=at(7), ld_y=20), dict(ld_x=20, y=at(13), ld_y=20), dict(ld_x=20, y=at(-7 - 20 * 10), ld_y=20),
                dict(y=apart(1)), dict(y=apart(2)), dict(pre=apart(2)), dict(pre=apart(4)), dict(pre=apart(3)), dict(y=apart(3), ld_y=9),
                dict(residual=at(0), y=at(0)), dict(rows=9, bias=NULL, ld_x=100, y=at(800 + 7), ld_y=8),
                dict(rows=1, y=at(7), ws=apart(6))):
        assert call(L.amq_linear, args, **bad) == INVALID, bad


def test_linear_backward(L):
    rows, k, n = 20, 8, 8
    need = L.amq_linear_backward_workspace_bytes(rows, k, n, BF16)
    args = dict(dy=apart(0), ld_dy=8, x=apart(1), ld_x=8, W=apart(2), ld_w=8, pre=apart(3), ld_pre=8, rows=rows, k=k, n=n, type=BF16, act=1, dx=apart(4),
                ld_dx=8, dW=apart(5), ld_dw=8, dbias=apart(6), ws=apart(7), bytes=need, stream=None)
    for bad in (dict(dx=apart(0)), dict(dx=apart(1)), dict(dx=apart(2)), dict(dx=apart(3)), dict(dW=apart(0)), dict(dW=apart(1)), dict(dW=apart(2)),
                dict(dW=apart(3)), dict(dW=apart(4)), dict(dbias=apart(4)), dict(dbias=apart(5)), dict(dbias=apart(0)), dict(dbias=apart(3))):
        assert call(L.amq_linear_backward, args, **bad) == INVALID, bad


def test_layer_norm(L):
    args = dict(x=at(0), ld_x=8, rows=4, n=8, type=F32, weight=apart(1), bias=apart(2), param_type=F32, eps=C.c_float(1e-5), y=apart(3), ld_y=8,
                mean=apart(4), rstd=apart(5), stream=None)
    for bad in (dict(y=at(1)), dict(y=at(31)), dict(y=at(-31)), dict(y=at(0), ld_y=9), dict(y=apart(1)), dict(y=apart(2)), dict(mean=at(31)),
                dict(mean=apart(3)), dict(rstd=apart(4)), dict(rstd=apart(1)), dict(ld_x=20, y=at(7), ld_y=20)):
        assert call(L.amq_layer_norm, args, **bad) == INVALID, bad
    need = L.amq_layer_norm_backward_workspace_bytes(4, 8)
    args = dict(dy=apart(0), ld_dy=8, x=apart(1), ld_x=8, rows=4, n=8, type=F32, weight=apart(2), param_type=F32, mean=apart(3), rstd=apart(4), dx=apart(5),
                ld_dx=8, dweight=apart(6), dbias=apart(7), ws=apart(8), bytes=need, stream=None)
    for bad in (dict(dx=apart(0), ld_dx=9), dict(dx=apart(1), ld_dx=9), dict(dx=apart(2)), dict(dx=apart(3)), dict(dx=apart(4)), dict(dweight=apart(0)),
                dict(dweight=apart(2)), dict(dbias=apart(6)), dict(dbias=apart(5)), dict(dbias=apart(1)), dict(dweight=apart(4))):
        assert call(L.amq_layer_norm_backward, args, **bad) == INVALID, bad


def test_orthogonalize_without_steps(L):
    need = L.amq_orthogonalize_workspace_bytes(3, 8, 6, F32)
    coef = (C.c_float * 3)(3.4445, -4.775, 2.0315)
    args = dict(G=at(0), batch=3, stride=0, rows=8, cols=6, ld=6, type=F32, steps=0, coef=coef, eps=C.c_float(1e-7), out=apart(1), stride_out=0, ld_out=6,
                ws=apart(2), bytes=need, stream=None)
    for bad in (dict(out=at(1)), dict(out=at(143)), dict(out=at(-143)), dict(out=at(0), ld_out=7), dict(out=at(0), stride_out=50),
                dict(out=at(48)), dict(out=at(-96), stride_out=100)):
        assert call(L.amq_orthogonalize, args, **bad) == INVALID, bad


@pytest.mark.gpu
def test_columns_of_one_matrix_are_apart():
    """Operands and results side by side, above and below each other in one wider matrix, and with strides of their own, are taken as they are."""
    import torch
    import paper_1802_00150_amd as amq
    from train_util import DEV, rand
    rows, k, n = 90, 24, 40
    x, W, r = rand(1, rows, k).to(DEV), rand(2, n, k).to(DEV), rand(3, rows, n).to(DEV)
    plain = amq.linear(x, W, None, "silu", r)
    wide = torch.zeros(rows + n, 200, device=DEV)
    xs, rs, ys, ps, Ws = wide[:rows, 1:1 + k], wide[:rows, 30:30 + n], wide[:rows, 70:70 + n], wide[:rows, 110:110 + n], wide[rows:, 3:3 + k]
    xs.copy_(x), rs.copy_(r), Ws.copy_(W)
    assert torch.equal(amq.linear(xs, Ws, None, "silu", rs, out=ys, pre=ps), plain)
    assert torch.equal(xs, x) and torch.equal(rs, r) and torch.equal(Ws, W)
    # every other row of the same memory
    flat = torch.zeros(2 * rows, 64, device=DEV)
    even, odd = flat[::2, :k], flat[1::2, :n]
    even.copy_(x)
    assert torch.equal(amq.linear(even, W, out=odd), amq.linear(x, W)) and torch.equal(even, x)
    # different strides: the result between the operand's rows
    far = torch.zeros(rows * 400, device=DEV)
    xs = far.view(rows, 400)[:, 300:300 + k]
    xs.copy_(x)
    ys = far[:40].view(1, 40)
    assert torch.equal(amq.linear(xs[:1], W, out=ys), amq.linear(x[:1], W))
    y, mean, rstd = amq.layer_norm(x)
    wide[:rows, 1:1 + k].copy_(x)
    got = amq.layer_norm(wide[:rows, 1:1 + k], out=wide[:rows, 1 + k:1 + 2 * k])
    assert torch.equal(got[0], y) and torch.equal(got[1], mean)
    for out in (wide[:rows, 1:1 + k], x):
        with pytest.raises(amq.AmqError):
            amq.linear(out, torch.eye(k, device=DEV), out=out)
    with pytest.raises(amq.AmqError):
        amq.layer_norm(wide[:rows, 1:1 + k], out=wide[:rows, 2:2 + k])
    G = rand(4, 2, 30, 20).to(DEV)
    stack = torch.zeros(2, 30, 50, device=DEV)
    stack[:, :, :20].copy_(G)
    for steps in (0, 3):
        assert torch.equal(amq.orthogonalize(stack[:, :, :20], steps=steps, out=stack[:, :, 25:45]), amq.orthogonalize(G, steps=steps))
        assert torch.equal(amq.orthogonalize(G.clone(), steps=steps, out=None), amq.orthogonalize(G, steps=steps))
    again = G.clone()
    assert torch.equal(amq.orthogonalize(again, steps=0, out=again), amq.orthogonalize(G, steps=0))
    shifted = torch.zeros(2 * 30 * 20 + 7, device=DEV)
    a, b = shifted[:1200].view(2, 30, 20), shifted[7:].view(2, 30, 20)
    a.copy_(G)
    assert torch.equal(amq.orthogonalize(a, steps=3, out=b), amq.orthogonalize(G, steps=3))
    a.copy_(G)
    with pytest.raises(amq.AmqError):
        amq.orthogonalize(a, steps=0, out=b)
