"""Refusals of the calls around a residual block (norms, embedding, gradient clipping): every check runs on the host before
any GPU work, so the placeholder pointers below are never dereferenced."""

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


def _n(C, kind=1, eps=1e-5, **at):
    f = {k: A * v for k, v in at.items()}
    return C.csrt_norm(kind, eps, f.get("weight"), f.get("bias"), f.get("mean"), f.get("rstd"), f.get("dweight"), f.get("dbias"))


WS = ctypes.c_void_p(A * 100)
BIG = ctypes.c_size_t(1 << 40)


def test_block_norm_fwd_refuses(C):
    L = C.lib()
    y, g, r, h, v = (_m(C, k, 8, 16) for k in (1, 2, 3, 4, 5))

    def call(y=y, post=_n(C, weight=10), g=g, act=1, r=r, rs=1.0, pre=_n(C, weight=11), h=h, v=v):
        return L.csrt_block_norm_fwd(y, post, g, act, r, F(rs), pre, h, v, None)

    _expect(C, call(y=None, r=None, post=None, g=None), "y and r are both NULL")
    _expect(C, call(h=None, v=None, pre=None), "h and v are both NULL")
    _expect(C, call(y=None, g=None), "post and gate need y")
    _expect(C, call(y=None, post=None), "post and gate need y")
    _expect(C, call(pre=None), "pre and v go together")
    _expect(C, call(v=None), "pre and v go together")
    _expect(C, call(act=3), "unknown gate activation 3")
    _expect(C, call(rs=float("nan")), "r_scale must be finite")
    _expect(C, call(g=_m(C, 2, 8, 15)), "gate is 8 x 15, must be 8 x 16")
    _expect(C, call(v=_m(C, 5, 9, 16)), "v is 9 x 16")
    _expect(C, call(r=_m(C, 3, 8, 16, ld=15)), "r: bad ld")
    _expect(C, call(h=_m(C, None, 8, 16)), "h: data is NULL")
    _expect(C, call(g=_m(C, 2, 8, 16, dtype=2)), "gate has another type")
    _expect(C, call(h=_m(C, 4, 8, 16, dtype=0)), "h has another type")
    _expect(C, call(r=_m(C, 3, 8, 16, dtype=2), h=_m(C, 4, 8, 16, dtype=2)), "float32 or of the block's type")
    _expect(C, call(post=_n(C, kind=3)), "post: unknown norm 3")
    _expect(C, call(pre=_n(C, eps=0.0)), "pre: eps must be")
    _expect(C, call(pre=_n(C, eps=float("inf"))), "pre: eps must be")
    bad = _n(C)
    bad.weight = A * 10 + 2
    _expect(C, call(post=bad), "post is not aligned")
    _expect(C, call(h=_m(C, 1, 8, 16)), "h overlaps y")
    _expect(C, call(v=_m(C, 4, 8, 16)), "h overlaps v")
    _expect(C, call(v=_m(C, 2, 8, 16)), "v overlaps gate")
    _expect(C, call(v=_m(C, 3, 8, 16)), "v overlaps r")
    _expect(C, call(h=C.csrt_mat(A * 3 + 2, 8, 16, 16, 1)), "h overlaps r")
    _expect(C, call(pre=_n(C, rstd=4)), "h overlaps pre.rstd")
    _expect(C, call(pre=_n(C, weight=5)), "v overlaps pre.weight")
    _expect(C, call(post=_n(C, kind=2, mean=12, rstd=12)), "post.mean overlaps post.rstd")
    _expect(C, call(post=_n(C, rstd=1)), "post.rstd overlaps y")
    _expect(C, call(r=None, post=_n(C, weight=4)), "h overlaps post.weight")
    _expect(C, call(y=None, post=None, g=None, h=None, pre=_n(C, weight=5)), "v overlaps pre.weight")


def test_block_norm_bwd_refuses(C):
    L = C.lib()
    dv, dh, h, y, g, dr, dy, dg = (_m(C, k, 8, 16) for k in range(1, 9))
    P, Q = _n(C, kind=2, weight=10, mean=12, rstd=13, dweight=14, dbias=15), _n(C, kind=1, weight=11, rstd=16, dweight=17)

    def call(dv=dv, dh=dh, h=h, pre=P, y=y, post=Q, g=g, act=1, rs=1.0, dr=dr, dy=dy, dg=dg, ws=WS, n=BIG):
        return L.csrt_block_norm_bwd(dv, dh, h, pre, y, post, g, act, F(rs), 0, dr, dy, dg, ws, n, None)

    _expect(C, call(dv=None, dh=None, pre=None), "dv and dh are both NULL")
    _expect(C, call(dv=None), "pre and dv go together")
    _expect(C, call(h=None), "pre needs h")
    _expect(C, call(dy=None), "post and gate need dy")
    _expect(C, call(g=None), "dgate needs gate")
    _expect(C, call(y=None), "post and dgate need y")
    _expect(C, call(act=-1), "unknown gate activation")
    _expect(C, call(rs=float("inf")), "r_scale")
    _expect(C, call(dy=_m(C, 7, 8, 17)), "dy is 8 x 17")
    _expect(C, call(dr=_m(C, 6, 8, 16, dtype=0)), "another type")
    _expect(C, call(dy=_m(C, 7, 8, 16, dtype=0)), "dy has another type")
    _expect(C, call(pre=_n(C, kind=2, rstd=13)), "pre: the backward pass needs mean")
    _expect(C, call(post=_n(C, kind=1)), "post: the backward pass needs rstd")
    _expect(C, call(dr=_m(C, 3, 8, 16)), "dr overlaps h")
    _expect(C, call(dy=_m(C, 6, 8, 16)), "dr overlaps dy")
    _expect(C, call(dg=_m(C, 5, 8, 16)), "dgate overlaps gate")
    _expect(C, call(post=_n(C, kind=1, rstd=16, dweight=14)), "post.dweight overlaps pre.dweight")
    _expect(C, call(post=_n(C, kind=1, rstd=16, dweight=13)), "post.dweight overlaps pre.rstd")
    _expect(C, call(post=_n(C, kind=1, rstd=16, dbias=2)), "post.dbias overlaps dh")
    _expect(C, call(dh=None, post=_n(C, kind=1, rstd=16, dweight=6)), "dr overlaps post.dweight")
    _expect(C, call(ws=None), "workspace is NULL")
    _expect(C, call(ws=ctypes.c_void_p(A * 100 + 8)), "not 256-byte aligned")
    _expect(C, call(n=ctypes.c_size_t(256)), "workspace has 256 bytes", C.CSRT_ERR_WORKSPACE)
    n = ctypes.c_size_t(0)
    _expect(C, L.csrt_block_norm_workspace_bytes(-1, 4, ctypes.byref(n)), "negative")
    _expect(C, L.csrt_block_norm_workspace_bytes(4, 4, None), "bytes is NULL")


def test_embed_refuses(C):
    L = C.lib()
    table, x, tok = _m(C, 1, 100, 16, dtype=0), _m(C, 2, 16, 24), ctypes.c_void_p(A * 3)

    def fwd(table=table, tok=tok, scale=1.0, x=x, ws=WS, n=BIG):
        return L.csrt_embed_fwd(table, tok, F(scale), x, ws, n, None)

    def bwd(dx=x, tok=tok, scale=1.0, dtable=table, ws=WS, n=BIG):
        return L.csrt_embed_bwd(dx, tok, F(scale), 0, dtable, ws, n, None)

    _expect(C, fwd(table=None), "table is NULL")
    _expect(C, fwd(x=_m(C, 2, 15, 24)), "x is 15 x 24, must be 16 x 24")
    _expect(C, fwd(tok=None), "tokens is NULL")
    _expect(C, fwd(tok=ctypes.c_void_p(A * 3 + 2)), "tokens is not aligned")
    _expect(C, fwd(tok=ctypes.c_void_p(A * 2 + 64)), "tokens overlap x")
    _expect(C, fwd(scale=float("nan")), "scale must be finite")
    _expect(C, fwd(x=_m(C, 1, 16, 24)), "x overlaps table")
    _expect(C, fwd(ws=None), "workspace is NULL")
    _expect(C, fwd(ws=ctypes.c_void_p(A * 100 + 4)), "not 256-byte aligned")
    _expect(C, fwd(n=ctypes.c_size_t(4)), "workspace has 4 bytes", C.CSRT_ERR_WORKSPACE)
    _expect(C, bwd(dtable=_m(C, 1, 100, 17, dtype=0)), "dtable is 100 x 17, must be 100 x 16")
    _expect(C, bwd(tok=None), "tokens is NULL")
    _expect(C, bwd(tok=ctypes.c_void_p(A * 1 + 64)), "tokens overlap dtable")
    _expect(C, bwd(dtable=_m(C, 2, 100, 16)), "dtable overlaps dx")
    _expect(C, bwd(n=ctypes.c_size_t(4)), "workspace has 4 bytes", C.CSRT_ERR_WORKSPACE)
    n = ctypes.c_size_t(0)
    _expect(C, L.csrt_embed_workspace_bytes(1, 1, -1, ctypes.byref(n)), "negative")
    # nothing to look up, nothing to write
    assert fwd(x=_m(C, None, 16, 0), tok=None) == 0
    assert bwd(dtable=_m(C, None, 0, 16)) == 0


def test_grad_clip_refuses(C):
    L = C.lib()

    def mats(*m):
        a = (C.csrt_mat * len(m))()
        for k, v in enumerate(m):
            a[k] = v
        return a

    g, o = mats(_m(C, 1, 8, 16, dtype=0), _m(C, 2, 1, 16)), mats(_m(C, 3, 8, 16), _m(C, 4, 1, 16))
    norm = ctypes.c_void_p(A * 9)

    def call(g=g, count=2, max_norm=1.0, o=o, norm=norm, ws=WS, n=BIG):
        return L.csrt_grad_clip(g, count, F(max_norm), o, norm, ws, n, None)

    _expect(C, call(count=-1), "count is negative")
    _expect(C, call(g=None), "g is NULL")
    _expect(C, call(norm=None), "norm is NULL")
    _expect(C, call(norm=ctypes.c_void_p(A * 9 + 1)), "norm is not aligned")
    _expect(C, call(norm=ctypes.c_void_p(A * 2 - 4)), "norm overlaps g[1]")
    _expect(C, call(norm=ctypes.c_void_p(A * 3 + 8)), "norm overlaps out[0]")
    _expect(C, call(o=mats(_m(C, 3, 8, 15), _m(C, 4, 1, 16))), "out is 8 x 15, must be 8 x 16")
    _expect(C, call(g=mats(_m(C, 1, 8, 16, dtype=9), _m(C, 2, 1, 16))), "unknown dtype")
    _expect(C, call(o=mats(_m(C, 1, 8, 16), _m(C, 4, 1, 16))), "out[0] overlaps g[0]")
    for bad in (0.0, -1.0, float("inf"), float("nan")):
        _expect(C, call(max_norm=bad), "max_norm must be")
    _expect(C, call(ws=None), "workspace is NULL")
    _expect(C, call(n=ctypes.c_size_t(4)), "workspace has 4 bytes", C.CSRT_ERR_WORKSPACE)
    _expect(C, L.csrt_grad_norm(g, 2, None, WS, BIG, None), "norm is NULL")
    _expect(C, L.csrt_grad_workspace_bytes(None), "bytes is NULL")


def test_python_side_refuses(C):
    with pytest.raises(ValueError, match="unknown norm"):
        C.Norm("batch")
    with pytest.raises(ValueError, match="unknown gate"):
        C._gate("tanh")
    torch = pytest.importorskip("torch")
    with pytest.raises(ValueError, match="weight must be a contiguous float32 CUDA tensor"):
        C.Norm("rms", weight=torch.ones(4))
    with pytest.raises(ValueError, match="tokens must be"):
        C.embed_fwd(None, torch.zeros(4, dtype=torch.int32), torch.zeros(4, 4), None)
    with pytest.raises(ValueError, match="tensor 0 must be"):
        C.TensorList([torch.zeros(4, 4, 4).transpose(0, 1)])


def test_lookups_need_the_status_words_alone(C):
    """Whatever the number of tokens and features; the gradient asks for more."""
    L, n = C.lib(), ctypes.c_size_t(0)
    assert L.csrt_embed_workspace_bytes(100, 4096, 0, ctypes.byref(n)) == 0
    few = n.value
    assert L.csrt_embed_workspace_bytes(7, 2 ** 31 - 1, 0, ctypes.byref(n)) == 0 and n.value == few
    table, x, tok = _m(C, 1, 100, 16, dtype=0), _m(C, 2, 16, 24), ctypes.c_void_p(A * 3)
    _expect(C, L.csrt_embed_fwd(table, tok, F(1), x, WS, ctypes.c_size_t(few - 1), None), f"needs {few}", C.CSRT_ERR_WORKSPACE)
    _expect(C, L.csrt_embed_bwd(x, tok, F(1), 0, table, WS, ctypes.c_size_t(few), None), f"workspace has {few} bytes",
            C.CSRT_ERR_WORKSPACE)


def test_embed_workspace_sizes_do_not_wrap(C):
    """Sizes that no call takes are refused."""
    L, n = C.lib(), ctypes.c_size_t(0)
    assert L.csrt_embed_workspace_bytes(9, 2 ** 20, 2 ** 20, ctypes.byref(n)) == 0 and n.value > 2 ** 42
    for d, max_n in ((2 ** 31 - 1, 2 ** 31 - 1), (2 ** 20 + 1, 2 ** 20), (2 ** 31 - 1, 2 ** 30)):
        _expect(C, L.csrt_embed_workspace_bytes(9, d, max_n, ctypes.byref(n)), "too large")
