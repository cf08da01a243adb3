"""Refusals of the dense-layer calls and of the orthogonalised update: every check runs on the host before any GPU
work, so the placeholder pointers below are never dereferenced."""

import ctypes

import pytest

F = ctypes.c_float
A = 1 << 20   # placeholder arrays a megabyte apart


@pytest.fixture(scope="module")
def C():
    from paper_1905_07931_gb300 import build
    build.build()
    from paper_1905_07931_gb300 import csrtrain
    csrtrain.lib()
    return csrtrain


def _expect(C, rc, fragment, code=None):
    assert rc == (C.CSRT_ERR_ARG if code is None else code), rc
    msg = C.lib().csrt_last_error().decode()
    assert fragment in msg, msg


def _m(C, at, rows, cols, ld=None, dtype=1):
    return C.csrt_mat(A * at if at is not None else None, rows, cols, cols if ld is None else ld, dtype)


WS = ctypes.c_void_p(A * 100)
BIG = ctypes.c_size_t(1 << 40)


def test_dense_fwd_refuses(C):
    L = C.lib()
    w, x, y = _m(C, 1, 8, 16), _m(C, 2, 16, 4), _m(C, 3, 8, 4)

    def call(w=w, x=x, y=y, act=0, r=None, z=None, ws=WS, n=BIG):
        return L.csrt_dense_fwd(w, x, None, act, r, z, y, ws, n, None)

    _expect(C, L.csrt_dense_fwd(None, x, None, 0, None, None, y, WS, BIG, None), "w is NULL")
    _expect(C, call(x=_m(C, 2, 15, 4)), "x is 15 x 4, must be 16 x 4")
    _expect(C, call(y=_m(C, 3, 8, 5)), "y is 8 x 5")
    _expect(C, call(w=_m(C, 1, -1, 16)), "negative size")
    _expect(C, call(x=_m(C, 2, 16, 4, ld=3)), "bad ld")
    _expect(C, call(x=_m(C, None, 16, 4)), "data is NULL")
    _expect(C, call(x=_m(C, 2, 16, 4, dtype=7)), "unknown dtype")
    _expect(C, call(x=_m(C, 2, 16, 4, dtype=2)), "one 16-bit type")
    _expect(C, call(w=_m(C, 1, 8, 16, dtype=0), x=_m(C, 2, 16, 4, dtype=0)), "one 16-bit type")
    _expect(C, call(y=_m(C, 3, 8, 4, dtype=2)), "float32 or of the operands' type")
    _expect(C, call(act=9), "unknown activation")
    _expect(C, call(r=_m(C, 4, 8, 4, dtype=0)), "residual must have y's type")
    _expect(C, call(z=_m(C, 4, 8, 4, dtype=0)), "z must have w's type")
    _expect(C, call(y=_m(C, 2, 8, 4)), "y overlaps an operand")
    _expect(C, call(z=_m(C, 3, 8, 4)), "z overlaps")
    r = C.csrt_mat(A * 3 + 16, 8, 4, 4, 1)   # half over y
    _expect(C, call(r=r), "y overlaps residual")
    odd = C.csrt_mat(A * 2 + 1, 16, 4, 4, 1)
    _expect(C, call(x=odd), "not aligned to its type")
    _expect(C, call(ws=None), "workspace is NULL")
    _expect(C, call(ws=ctypes.c_void_p(A * 100 + 16)), "not 256-byte aligned")
    _expect(C, call(n=ctypes.c_size_t(1024)), "workspace has 1024 bytes", C.CSRT_ERR_WORKSPACE)


def test_dense_backward_refuses(C):
    L = C.lib()
    w, dy, dx = _m(C, 1, 8, 16), _m(C, 2, 8, 4), _m(C, 3, 16, 4)
    z = _m(C, 4, 16, 4)
    _expect(C, L.csrt_dense_bwd_x(w, dy, None, 1, None, dx, WS, BIG, None), "needs z_below")
    _expect(C, L.csrt_dense_bwd_x(w, dy, _m(C, 4, 8, 4), 1, None, dx, WS, BIG, None), "z_below is 8 x 4")
    _expect(C, L.csrt_dense_bwd_x(w, dy, z, 1, None, _m(C, 4, 16, 4), WS, BIG, None), "dx overlaps z_below")
    _expect(C, L.csrt_dense_bwd_x(w, dy, z, 4, None, dx, WS, BIG, None), "unknown activation")
    _expect(C, L.csrt_dense_bwd_x(w, _m(C, 2, 9, 4), None, 0, None, dx, WS, BIG, None), "dy is 9 x 4")
    x, dw = _m(C, 3, 16, 4), _m(C, 5, 8, 16, dtype=0)
    _expect(C, L.csrt_dense_bwd_w(dy, _m(C, 3, 16, 5), 0, dw, None, WS, BIG, None), "x is 16 x 5")
    _expect(C, L.csrt_dense_bwd_w(dy, x, 0, _m(C, 5, 16, 8, dtype=0), None, WS, BIG, None), "dw is 16 x 8")
    _expect(C, L.csrt_dense_bwd_w(dy, x, 0, _m(C, 3, 8, 16), None, WS, BIG, None), "dw overlaps an operand")
    _expect(C, L.csrt_dense_act_bwd(dy, None, 1, _m(C, 6, 8, 4), None), "z is NULL")
    _expect(C, L.csrt_dense_act_bwd(dy, None, 0, _m(C, 6, 8, 5), None), "dpre is 8 x 5")
    _expect(C, L.csrt_dense_update(_m(C, 1, 8, 16), dw, F(0.1), F(0), None, None), "w must be float32")
    wf = _m(C, 7, 8, 16, dtype=0)
    _expect(C, L.csrt_dense_update(wf, dw, F(-0.1), F(0), None, None), "finite and >= 0")
    _expect(C, L.csrt_dense_update(wf, dw, F(float("nan")), F(0), None, None), "finite and >= 0")
    _expect(C, L.csrt_dense_update(wf, wf, F(0.1), F(0), None, None), "w overlaps d")


def test_empty_dense_calls_do_nothing(C):
    L = C.lib()
    w, y = _m(C, 1, 0, 16), _m(C, 3, 0, 4)
    assert L.csrt_dense_fwd(w, _m(C, 2, 16, 4), None, 0, None, None, y, WS, BIG, None) == 0
    assert L.csrt_dense_fwd(_m(C, 1, 8, 16), _m(C, None, 16, 0), None, 0, None, None, _m(C, None, 8, 0), WS, BIG, None) == 0
    assert L.csrt_dense_act_bwd(_m(C, 1, 0, 4), None, 0, _m(C, 2, 0, 4), None) == 0


def test_orthogonalize_refuses(C):
    L = C.lib()
    g, o = _m(C, 1, 8, 16, dtype=0), _m(C, 2, 8, 16)
    mom = ctypes.c_void_p(A * 3)

    def call(g=g, gs=128, batch=1, mom=mom, beta=0.9, steps=5, eps=1e-7, scale=1.0, o=o, os=128, ws=WS, n=BIG):
        return L.csrt_orthogonalize(g, gs, batch, mom, F(beta), 1, steps, F(eps), F(scale), o, os, ws, n, None)

    _expect(C, call(batch=-1), "batch must be")
    _expect(C, call(batch=70000), "batch must be")
    _expect(C, call(g=_m(C, 1, 8, 16, dtype=2)), "g must be float32 or bfloat16")
    _expect(C, call(o=_m(C, 2, 16, 8)), "o is 16 x 8, must be 8 x 16")
    _expect(C, call(g=_m(C, 1, 8, 16, ld=15, dtype=0)), "bad ld")
    _expect(C, call(g=_m(C, 1, 65536, 65536, dtype=0), o=_m(C, 2, 65536, 65536)), "bad size")
    _expect(C, call(beta=1.0), "beta must be in")
    _expect(C, call(beta=float("nan")), "beta must be in")
    _expect(C, call(eps=0.0), "eps must be")
    _expect(C, call(scale=float("inf")), "scale must be finite")
    _expect(C, call(steps=33), "steps must be")
    _expect(C, call(steps=-1), "steps must be")
    _expect(C, call(batch=2, os=100), "matrices of o overlap")
    _expect(C, call(o=_m(C, 1, 8, 16)), "o overlaps g")
    _expect(C, call(mom=ctypes.c_void_p(A * 2)), "momentum overlaps")
    _expect(C, call(ws=None), "workspace is NULL")
    _expect(C, call(n=ctypes.c_size_t(4096)), "workspace has 4096 bytes", C.CSRT_ERR_WORKSPACE)
    n = ctypes.c_size_t(0)
    assert L.csrt_orthogonalize_workspace_bytes(3, 300, 784, ctypes.byref(n)) == 0 and n.value > 3 * 300 * 784 * 6
    _expect(C, L.csrt_orthogonalize_workspace_bytes(1, 1 << 16, 1 << 16, ctypes.byref(n)), "2^31")
    _expect(C, L.csrt_dense_workspace_bytes(-1, 3, 3, ctypes.byref(n)), "negative")


def test_the_largest_number_of_rows_is_taken(C):
    """2^31 - 1 rows pass the check of the leading dimension (the call then fails on the output's shape)."""
    L, m = C.lib(), 2 ** 31 - 1
    w, x = _m(C, 1, m, 1), _m(C, 2, 1, 4)
    _expect(C, L.csrt_dense_fwd(w, x, None, 0, None, None, _m(C, 3, 8, 4), WS, BIG, None), f"y is 8 x 4, must be {m} x 4")
    _expect(C, L.csrt_dense_fwd(_m(C, 1, m, 1, ld=1 << 10), x, None, 0, None, None, _m(C, 3, 8, 4), WS, BIG, None), "w: bad ld")


def test_bias_and_its_gradient_are_checked(C):
    """float32 vectors off their alignment, or over a matrix that the call writes (db also over one that it reads)."""
    L, vp = C.lib(), ctypes.c_void_p
    w, x, y, z = _m(C, 1, 8, 16), _m(C, 2, 16, 4), _m(C, 3, 8, 4), _m(C, 4, 8, 4)

    def fwd(bias, y=y):
        return L.csrt_dense_fwd(w, x, vp(bias), 0, None, z, y, WS, BIG, None)

    _expect(C, fwd(A * 9 + 2), "bias is not aligned")
    _expect(C, fwd(A * 3 + 32), "bias overlaps y")
    _expect(C, fwd(A * 4 - 16), "bias overlaps z")
    _expect(C, fwd(A * 3 + 64 * 7 + 4, y=_m(C, 3, 8, 4, ld=32)), "bias overlaps y")
    # beside y's rows, or after its last one, it is no overlap: the call goes on to the next check, which this y fails
    for at in (A + 8, A + 32, A + 64 * 7 + 8):
        _expect(C, fwd(at, y=_m(C, 1, 8, 4, ld=32)), "y overlaps an operand")
    dy, xx, dw = _m(C, 1, 8, 4), _m(C, 2, 16, 4), _m(C, 5, 8, 16, dtype=0)

    def bwd(db):
        return L.csrt_dense_bwd_w(dy, xx, 0, dw, vp(db), WS, BIG, None)

    _expect(C, bwd(A * 9 + 1), "db is not aligned")
    _expect(C, bwd(A * 5 + 128), "db overlaps dw")
    _expect(C, bwd(A * 1 + 32), "db overlaps dy")
    _expect(C, bwd(A * 2 - 4), "db overlaps x")
