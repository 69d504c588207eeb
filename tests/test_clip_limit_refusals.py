"""Argument validation of the clipping's entry with a limit of binary64 (no GPU)."""
import ctypes as C

from test_recurrent_refusals import apart
from test_train_refusals import F32, INVALID, L, NULL  # noqa: F401


def test_clip_gradients_double(L):  # noqa: F811
    p = (C.c_void_p * 2)(apart(0).value, apart(1).value)
    need = L.amq_clip_gradients_workspace_bytes(2)

    def run(max_norm=1.0, norm=apart(9), out=p, sizes=(10, 20), bytes=need):
        return L.amq_clip_gradients_double(2, p, (C.c_int64 * 2)(*sizes), (C.c_int * 2)(F32, F32), max_norm, out, norm, apart(10), bytes, None)
    # (the second: a limit below 0 that binary32 would round to -0)
    for bad in (dict(max_norm=-1.0), dict(max_norm=-1e-60), dict(max_norm=float("nan")), dict(norm=NULL), dict(sizes=(-1, 3)), dict(bytes=need - 1), dict(norm=apart(1)),
                dict(out=(C.c_void_p * 2)(apart(1).value, apart(0).value))):
        assert run(**bad) == INVALID, bad
