"""Argument validation of the recurrent block's operators at the C ABI, which precedes any launch (no GPU)."""
import ctypes as C

from test_train_refusals import BF16, F16, F32, INVALID, L, NULL, ODD, P, UNSUPPORTED, call  # noqa: F401


def apart(i):  # the i-th of many buffers that do not meet
    return C.c_void_p(0x100000000 + i * 0x10000000)


def at(i, entry, size=4):  # `entry` elements behind the i-th buffer's begin
    return C.c_void_p(0x100000000 + i * 0x10000000 + entry * size)


def recurrence(steps=5, B=3, n=8, type=F32, **changed):
    a = dict(gate=apart(0), gs=B * n, gb=n, x=apart(1), xs=B * n, xb=n, steps=steps, B=B, n=n, type=type, mode=0, lengths=apart(2), h0=apart(3),
             hs=apart(4), ys=B * n, yb=n, h_last=apart(5), states=apart(6), ws=NULL, bytes=0, stream=None)
    assert not set(changed) - set(a)
    return dict(a, **changed)


def test_linear_recurrence(L):
    f = L.amq_linear_recurrence
    for bad in (dict(gate=NULL), dict(x=NULL), dict(hs=NULL), dict(steps=0), dict(B=0), dict(n=-1), dict(type=3), dict(mode=2), dict(mode=-1),
                dict(gs=-1), dict(xb=-1), dict(ys=-24), dict(gate=ODD), dict(x=ODD), dict(hs=ODD), dict(h0=ODD), dict(h_last=ODD), dict(states=ODD, steps=200),
                dict(lengths=C.c_void_p(0x10004)),
                # rows of the result that share entries
                dict(yb=7), dict(ys=23), dict(ys=0), dict(yb=0), dict(ys=8, yb=8), dict(ys=8, yb=39)):
        assert call(f, recurrence(**bad)) == INVALID, bad
    for bad in (dict(steps=(1 << 24) + 1), dict(B=(1 << 22) + 1), dict(n=(1 << 20) + 1), dict(B=1 << 20, n=1 << 11), dict(gs=(1 << 36) + 1), dict(yb=(1 << 36) + 1)):
        assert call(f, recurrence(**bad)) == UNSUPPORTED, bad


def test_linear_recurrence_overlaps(L):
    f = L.amq_linear_recurrence
    last = 5 * 3 * 8 - 1
    for bad in (dict(hs=apart(0)), dict(hs=apart(1)), dict(hs=at(0, last)), dict(hs=at(1, -last)), dict(hs=apart(3)), dict(hs=apart(2)), dict(hs=apart(5)),
                dict(h_last=apart(0)), dict(h_last=at(1, last)), dict(h_last=at(3, 1)), dict(h_last=at(3, -23)), dict(h_last=apart(2)),
                dict(states=apart(3), steps=200), dict(states=at(5, 23), steps=200), dict(states=at(4, 200 * 24 - 1), steps=200),
                # columns of one wide projection that meet: by rows in order, and with the batch outside
                dict(gate=at(0, 0), gs=72, gb=24, x=at(0, 8), xs=72, xb=24, hs=at(0, 15), ys=72, yb=24),
                dict(gate=at(0, 0), gs=24, gb=120, x=at(0, 8), xs=24, xb=120, hs=at(0, 15), ys=24, yb=120),
                # a slice of the steps and entries of a larger buffer
                dict(gate=at(0, 0), gs=300, gb=24, hs=at(0, 7), ys=300, yb=24), dict(gate=at(0, 0), gs=300, gb=24, hs=at(0, 300 * 4 + 48 + 7), ys=300, yb=24),
                # other strides than the operand's
                dict(gate=at(0, 0), gs=300, gb=24, hs=at(0, 1200), ys=24, yb=8),
                # a broadcast operand
                dict(gate=at(0, 0), gs=0, gb=0, hs=at(0, 7)), dict(x=at(0, 0), xs=24, xb=0, hs=at(0, 24 * 4 + 7))):
        assert call(f, recurrence(**bad)) == INVALID, bad


def test_linear_recurrence_backward(L):
    B, n = 3, 8
    def args(steps=5, **changed):
        a = dict(dhs=apart(0), ds=B * n, db=n, gate=apart(1), gs=B * n, gb=n, x=apart(2), xs=B * n, xb=n, steps=steps, B=B, n=n, type=F32, mode=0, lengths=apart(3),
                 h0=apart(4), states=apart(5), dh_last=apart(6), dgate=apart(7), rs=B * n, rb=n, dx=apart(8), qs=B * n, qb=n, dh0=apart(9), ws=NULL, bytes=0, stream=None)
        assert not set(changed) - set(a)
        return dict(a, **changed)
    f = L.amq_linear_recurrence_backward
    for bad in (dict(dhs=NULL), dict(gate=NULL), dict(x=NULL), dict(dgate=NULL), dict(dx=NULL), dict(states=NULL, steps=129), dict(type=4), dict(mode=3),
                dict(steps=0), dict(ds=-1), dict(rb=7), dict(qs=23), dict(qb=0), dict(dh0=ODD), dict(dh_last=ODD), dict(states=ODD),
                dict(dgate=apart(0)), dict(dgate=apart(1)), dict(dgate=apart(2)), dict(dx=apart(0)), dict(dx=apart(1)), dict(dx=apart(2)), dict(dx=apart(7)),
                dict(dx=at(7, 119)), dict(dgate=apart(4)), dict(dgate=apart(3)), dict(dx=apart(6)), dict(dh0=apart(6)), dict(dh0=apart(4)), dict(dh0=at(7, 119)),
                dict(dh0=at(2, 119)), dict(steps=129, dgate=at(5, 23)),
                # halves of one buffer that meet
                dict(dgate=at(7, 0), rs=48, rb=16, dx=at(7, 7), qs=48, qb=16)):
        assert call(f, args(**bad)) == INVALID, bad
    for bad in (dict(steps=(1 << 24) + 1), dict(ds=1 << 37), dict(qb=1 << 37)):
        assert call(f, args(**bad)) == UNSUPPORTED, bad


def test_block_norm(L):
    rows, n = 4, 8
    a = dict(x=apart(0), ld_x=n, residual=apart(1), ld_r=n, gate=apart(2), ld_g=n, rows=rows, n=n, type=BF16, residual_type=F32, param_type=F32, act=4,
             weight=apart(3), bias=apart(4), scale=apart(5), w2=apart(6), b2=apart(7), eps=C.c_float(1e-5), y=apart(8), ld_y=n, normed=apart(9), ld_n=n,
             stats=apart(10), stream=None)
    f = L.amq_block_norm
    for bad in (dict(x=NULL), dict(residual=NULL), dict(y=NULL), dict(type=3), dict(residual_type=F16), dict(param_type=F16), dict(act=1), dict(act=2), dict(act=6),
                dict(rows=0), dict(n=0), dict(ld_x=7), dict(ld_r=7), dict(ld_g=7), dict(ld_y=7), dict(ld_n=7), dict(eps=C.c_float(-1)),
                dict(eps=C.c_float(float("nan"))), dict(x=ODD), dict(residual=C.c_void_p(0x10002)), dict(y=C.c_void_p(0x10002)), dict(normed=ODD), dict(gate=ODD), dict(scale=ODD), dict(stats=ODD),
                dict(y=apart(0)), dict(y=apart(2)), dict(y=at(1, 1)), dict(y=apart(1), ld_y=9), dict(y=apart(9)), dict(y=apart(5)), dict(normed=apart(1)),
                dict(normed=apart(0)), dict(normed=apart(2)), dict(normed=apart(6)), dict(stats=apart(8)), dict(stats=apart(0)), dict(stats=at(9, 15)), dict(stats=apart(3))):
        assert call(f, a, **bad) == INVALID, bad
    assert call(f, a, n=16385, ld_x=20000, ld_r=20000, ld_g=20000, ld_y=20000, ld_n=20000) == UNSUPPORTED
    assert call(f, a, rows=1 << 31) == UNSUPPORTED


def test_block_norm_backward(L):
    rows, n = 4, 8
    need = L.amq_block_norm_backward_workspace_bytes(rows, n)
    assert need > 0 and need % 256 == 0 and L.amq_block_norm_backward_workspace_bytes(0, n) == 0 and L.amq_block_norm_backward_workspace_bytes(4, 16385) == 0
    a = dict(dy=apart(0), ld_dy=n, dnormed=apart(1), ld_dn=n, x=apart(2), ld_x=n, y=apart(3), ld_y=n, gate=apart(4), ld_g=n, rows=rows, n=n, type=BF16,
             residual_type=F32, param_type=F32, act=3, weight=apart(5), bias=apart(6), scale=apart(7), w2=apart(8), stats=apart(9), dx=apart(10), ld_dx=n,
             dresidual=apart(11), ld_dr=n, dgate=apart(12), ld_dg=n, dweight=apart(13), dbias=apart(14), dscale=apart(15), dw2=apart(16), db2=apart(17),
             ws=apart(18), bytes=need, stream=None)
    f = L.amq_block_norm_backward
    for bad in (dict(dy=NULL, dnormed=NULL), dict(x=NULL), dict(y=NULL), dict(stats=NULL), dict(dx=NULL), dict(gate=NULL), dict(type=9), dict(residual_type=F16),
                dict(param_type=F16), dict(act=5), dict(rows=-1), dict(ld_dy=7), dict(ld_dn=7), dict(ld_y=7), dict(ld_g=7), dict(ld_dx=7), dict(ld_dr=7),
                dict(ld_dg=7), dict(ws=NULL), dict(bytes=need - 1), dict(ws=C.c_void_p(0x10010)), dict(dscale=ODD), dict(dresidual=C.c_void_p(0x10002)),
                dict(dx=apart(2)), dict(dx=apart(0)), dict(dresidual=apart(0), ld_dr=9), dict(dresidual=at(0, 1)), dict(dresidual=apart(3)),
                dict(dgate=apart(4)), dict(dgate=apart(10)), dict(dweight=apart(5)), dict(dweight=at(14, 7)), dict(db2=apart(16)), dict(dscale=apart(9)),
                dict(dbias=apart(11)), dict(dw2=apart(0)), dict(dw2=apart(1))):
        assert call(f, a, **bad) == INVALID, bad
    assert call(f, a, n=16385, **{k: 20000 for k in a if k.startswith("ld_")}) == UNSUPPORTED


def test_clip_gradients(L):
    def run(tensors, sizes, types, out="in place", max_norm=1.0, norm=apart(9), ws=apart(10), bytes=None, count=None):
        n = len(tensors) if count is None else count
        pointers = (C.c_void_p * max(1, len(tensors)))(*tensors)
        results = pointers if out == "in place" else None if out is None else (C.c_void_p * max(1, len(out)))(*out)
        need = L.amq_clip_gradients_workspace_bytes(max(n, 0))
        return L.amq_clip_gradients(n, pointers, (C.c_int64 * max(1, len(sizes)))(*sizes), (C.c_int * max(1, len(types)))(*types), C.c_float(max_norm),
                                    results, norm, ws, need if bytes is None else bytes, None)
    assert L.amq_clip_gradients_workspace_bytes(-1) == 0 and L.amq_clip_gradients_workspace_bytes(0) > 0
    assert L.amq_clip_gradients_workspace_bytes(1000) > L.amq_clip_gradients_workspace_bytes(1)
    p = [apart(i).value for i in range(4)]
    types, sizes = [F32, BF16, F16, F32], [10, 20, 30, 40]
    for bad in (dict(count=-1), dict(max_norm=-1.0), dict(max_norm=float("nan")), dict(norm=NULL), dict(norm=ODD), dict(ws=NULL), dict(bytes=8), dict(ws=C.c_void_p(0x10010)),
                dict(norm=at(0, 9)), dict(norm=at(3, 39)), dict(out=[p[0], p[1], p[2], p[2]]), dict(out=[p[1], p[0], p[2], p[3]]), dict(out=[p[0] + 4, p[1], p[2], p[3]]),
                dict(out=[p[0], p[1], p[2], None]), dict(out=[p[0], p[1] + 1, p[2], p[3]]), dict(out=[p[0], p[0] + 36, p[2], p[3]])):
        assert run(p, sizes, types, **bad) == INVALID, bad
    assert run([p[0], p[1], p[2], p[3] + 1], sizes, types) == INVALID
    assert run([p[0], p[1], p[2], None], sizes, types) == INVALID
    assert run([p[0], p[1], p[0], p[3]], sizes, types) == INVALID       # the same memory scaled twice
    assert run(p, [10, -1, 30, 40], types) == INVALID
    assert run(p, sizes, [F32, BF16, F16, 3]) == INVALID
    assert run(p, [10, 20, 30, (1 << 40) + 1], types) == UNSUPPORTED
    assert run([], [], [], count=(1 << 20) + 1) in (INVALID, UNSUPPORTED)



def test_recurrence_workspaces(L):
    """None for one tile, for single tokens and where the channels fill the card by far; else 12 bytes for 64 channels of every tile and what they need
    beside it, whether batch entries count as channels or not."""
    for f in (L.amq_linear_recurrence_workspace_bytes, L.amq_linear_recurrence_backward_workspace_bytes):
        for type in (F32, BF16, F16):
            for steps, B, n in ((1, 1, 1), (128, 1, 1), (128, 256, 1024), (1000, 1 << 22, 1), (300, 1 << 20, 3), (1 << 24, 1 << 10, 1 << 17)):
                assert f(steps, B, n, type) == 0, (steps, B, n)
            need = f(1 << 24, 1, 64, type)
            assert need % 256 == 0 and 0 < need <= (1 << 17) * (64 * 12 + 4) + 8192
            assert f(20000, 4, 64, type) > 0
            for bad in ((0, 1, 1), (1, 0, 1), (1, 1, -1), ((1 << 24) + 1, 1, 1)):
                assert f(*bad, type) == 0
        assert f(1000, 1, 1, 3) == 0
