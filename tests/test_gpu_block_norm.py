"""The norms around a residual block against their definitions in float64.

Bounds, with u = 2^-24. A sum over d features passes through at most K = 64 + d / 1024 + 32 roundings (runs of 64, the
runs, the warps and blocks): off by K u sum |.|. Errors go through the formulas to first order with the error of each
operand; the gate's fast sigmoid is off by (4 + 1.2 |g|) 2^-23 of itself (the exponential's 2 + 1.173 |g| steps and the
quotient's two). Sums over n tokens pass through 320 + n / 32 roundings at most. Second-order terms are covered by a
factor 1.01 and 1e-30. The result is rounded once to its type: half a step, eps / 2.
"""

import math

import pytest

torch = pytest.importorskip("torch")

DT = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
U = 2.0 ** -24
EPS = 1e-5


@pytest.fixture(scope="module")
def C():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_1905_07931_gb300 import csrtrain
    csrtrain.lib()
    return csrtrain


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _mat(gen, rows, cols, dt, layout="tight", scale=1.0):
    """rows x cols values; layout: tight rows, "wide" (rows of a wider buffer, aligned), "odd" (base and rows off the
    16-byte grid). What surrounds them is NaN."""
    v = (torch.randn(rows, cols, generator=gen, device="cuda") * scale).to(dt)
    if layout == "tight":
        return v
    wide = (cols + 63) // 64 * 64 + 64 if layout == "wide" else cols + 5
    buf = torch.full((rows, wide), float("nan"), dtype=dt, device="cuda")
    view = buf[:, 0:cols] if layout == "wide" else buf[:, 3:3 + cols]
    view.copy_(v)
    return view


def _around(t):
    """The elements of a view's buffer that are not the view's, flattened."""
    buf = t._base
    if buf is None:
        return torch.empty(0, device="cuda")
    mask = torch.ones_like(buf, dtype=torch.bool)
    o = t.storage_offset() % buf.stride(0)
    mask[:, o:o + t.shape[1]] = False
    return buf[mask]


def _check(got, want, tol, name):
    dt = got.dtype
    tol = 1.01 * tol + torch.finfo(dt).eps / 2 * (want.abs() + 1.01 * tol) + (2.0 ** -25 if dt == torch.float16 else 0) + 1e-30
    bad = ~((got.double() - want).abs() <= tol)
    assert not bad.any(), (name, int(bad.sum()), float(((got.double() - want).abs() / tol).nan_to_num(1e30).max()))


def _sum_roundings(d):
    return 64 + d / 1024 + 32


def _sigmoid(g):
    return 0.5 * (1 + torch.tanh(0.5 * g))


def _gate(g, act):
    """a(g), a'(g) and their errors."""
    if act == "none":
        return g, torch.ones_like(g), 0 * g, 0 * g
    p = _sigmoid(g)
    e = (4 + 1.2 * g.abs()) * 2.0 ** -23
    ep = p * e + 1e-37
    if act == "sigmoid":
        return p, p * (1 - p), ep, ep + 3 * U * p
    return g * p, p * (1 + g * (1 - p)), g.abs() * (ep + U * p), ep * (1 + 2 * g.abs()) + 4 * U * p * (1 + g.abs())


def _vec(v, fill, d):
    return torch.full((d, 1), fill, dtype=torch.float64, device="cuda") if v is None else v.double()[:, None]


def _norm(x, ex, kind, w, b):
    """The norm of x, known within ex, with its statistics: (out, error), (mean, error), (rstd, error)."""
    d = x.shape[0]
    w, b = _vec(w, 1.0, d), _vec(b, 0.0, d)
    k = _sum_roundings(d)
    m = em = r = er = torch.zeros_like(x[:1])
    r = r + 1
    if kind == "layer":
        m = x.mean(0, keepdim=True)
        em = ex.mean(0, keepdim=True) + (k + 1) * U * x.abs().mean(0, keepdim=True)
    c = x - m
    ec = ex + em + U * c.abs()
    if kind != "scale":
        var = (c * c).mean(0, keepdim=True)
        ev = (2 * c.abs() * ec + ec * ec).mean(0, keepdim=True) + (k + 2) * U * var
        r = (var + EPS).rsqrt()
        er = r * (ev / (2 * (var + EPS)) + ev * ev / (var + EPS) ** 2 + 4 * U)
    out = c * r * w + b
    eo = w.abs() * (ec * r + c.abs() * er + ec * er + 2 * U * (c * r).abs()) + U * out.abs()
    return (out, eo), (m[0], em[0]), (r[0], er[0])


SHAPES = [(1, 1), (3, 5), (64, 33), (100, 1), (4096, 1), (784, 256), (1000, 777), (513, 32), (130, 2), (4096, 24),
          (9216, 40), (5000, 7), (2048, 300), (7, 2000), (264, 1024), (1056, 64), (12000, 9), (12000, 16), (20000, 5), (20000, 2),
          (70000, 1)]
# block type, stream type, post, pre, gate activation (None: no gate), biases, layout
FORMS = [("bf16", "bf16", "rms", "rms", "sigmoid", False, "tight"),
         ("f16", "f16", "layer", "layer", "silu", True, "odd"),
         ("bf16", "f32", "layer", "rms", "none", True, "wide"),
         ("f16", "f32", "scale", "layer", None, True, "tight"),
         ("f16", "f32", "rms", "layer", "silu", False, "odd"),
         ("bf16", "bf16", "scale", "rms", "sigmoid", True, "wide"),
         ("f32", "f32", "layer", "rms", "silu", True, "tight"),
         ("bf16", "bf16", "layer", "layer", None, False, "tight"),
         ("f16", "f16", "rms", "layer", "none", False, "wide")]


def _inputs(d, n, form, seed=None):
    tb, ts, post, pre, act, bias, layout = form
    gen = _gen(d * 131 + n * 17 if seed is None else seed)
    TB, TS = DT[tb], DT[ts]
    s = {"y": _mat(gen, d, n, TB, layout), "r": _mat(gen, d, n, TS, layout, 3.0),
         "g": _mat(gen, d, n, TB, layout, 2.0) if act is not None else None}
    s["y"].mul_(0.7).add_(0.3)
    for side in ("post", "pre"):
        s["w" + side] = 1 + 0.1 * torch.randn(d, generator=gen, device="cuda")
        s["b" + side] = 0.1 * torch.randn(d, generator=gen, device="cuda") if bias else None
    return gen, s


def _forward(s, post, pre, act, r_scale):
    """h, v and statistics with their errors."""
    (t, et), mp, rp = _norm(s["y"].double(), 0 * s["y"].double(), post, s["wpost"], s["bpost"])
    if s["g"] is not None:
        a, _, ea, _ = _gate(s["g"].double(), act)
        et = a.abs() * et + ea * (t.abs() + et) + U * (a * t).abs()
        t = a * t
    rr = r_scale * s["r"].double()
    h = rr + t
    eh = et + 2 * U * rr.abs() + U * h.abs()
    v, mq, rq = _norm(h, eh, pre, s["wpre"], s["bpre"])
    return (h, eh), v, mp, rp, mq, rq


@pytest.mark.gpu
@pytest.mark.parametrize("d,n", SHAPES)
@pytest.mark.parametrize("form", FORMS, ids=lambda f: "-".join(str(x) for x in f))
def test_forward(C, d, n, form):
    tb, ts, post, pre, act, bias, layout = form
    gen, s = _inputs(d, n, form)
    h, v = _mat(gen, d, n, DT[ts], layout), _mat(gen, d, n, DT[tb], layout)
    h.fill_(float("nan"))
    v.fill_(float("nan"))
    stat = {k: torch.full((n,), float("nan"), device="cuda") for k in ("mp", "rp", "mq", "rq")}
    P = C.Norm(post, s["wpost"], s["bpost"], EPS, stat["mp"], stat["rp"])
    Q = C.Norm(pre, s["wpre"], s["bpre"], EPS, stat["mq"], stat["rq"])
    rs = 0.9 if act != "silu" else -1.25
    C.block_norm_fwd(s["y"], s["r"], h, v, post=P, pre=Q, gate=s["g"], gate_act=act or "none", r_scale=rs)
    (hh, eh), (vv, ev), mp, rp, mq, rq = _forward(s, post, pre, act, rs)
    _check(h, hh, eh, "h")
    _check(v, vv, ev, "v")
    for name, kind, (want, err) in (("mp", post, mp), ("rp", post, rp), ("mq", pre, mq), ("rq", pre, rq)):
        if kind == "layer" or (kind == "rms" and name[0] == "r"):
            _check(stat[name], want, err, name)
        else:
            assert stat[name].isnan().all(), name   # not written
    for t in (h, v):
        assert _around(t).isnan().all()
    # in place over r, without statistics
    r2 = s["r"]
    P, Q = C.Norm(post, s["wpost"], s["bpost"], EPS), C.Norm(pre, s["wpre"], s["bpre"], EPS)
    v2, h2 = torch.full((d, n), float("nan"), dtype=v.dtype, device="cuda"), torch.empty((d, n), dtype=h.dtype, device="cuda")
    C.block_norm_fwd(s["y"], r2, h2, v2, post=P, pre=Q, gate=s["g"], gate_act=act or "none", r_scale=rs)
    _check(h2, hh, eh, "h into tight rows")
    _check(v2, vv, ev, "v into tight rows")
    v2 = _mat(gen, d, n, DT[tb], layout)
    C.block_norm_fwd(s["y"], r2, r2, v2, post=P, pre=Q, gate=s["g"], gate_act=act or "none", r_scale=rs)
    assert torch.equal(r2, h)
    assert torch.equal(v2, v)


def _backward(s, post, pre, act, r_scale, st):
    """Gradients and errors from the given statistics."""
    d, n = s["y"].shape
    kd, kn = _sum_roundings(d), 320 + n / 32

    def hat(x, side, kind):
        x = x.double()
        m = st["m" + side].double() if kind == "layer" else 0.0
        r = st["r" + side].double() if kind != "scale" else 1.0
        return (x - m) * r, 2 * U * ((x - m) * r).abs(), r

    def grad(dout, ed, xh, ex, r, kind, w):
        w = _vec(w, 1.0, d)
        g, eg = w * dout, w.abs() * ed + U * (w * dout).abs()
        if kind == "scale":
            return g, eg
        al = (g * xh).mean(0)
        eal = (g.abs() * ex + eg * xh.abs()).mean(0) + (kd + 3) * U * (g * xh).abs().mean(0)
        on = eon = 0 * al
        if kind == "layer":
            on, eon = g.mean(0), eg.mean(0) + (kd + 2) * U * g.abs().mean(0)
        q = g - xh * al - on
        eq = eg + ex * al.abs() + xh.abs() * eal + eon + 4 * U * (g.abs() + (xh * al).abs() + on.abs())
        return r * q, r * eq + U * (r * q).abs()

    hh, ehh, rh = hat(s["h"], "q", pre)
    yh, eyh, ry = hat(s["y"], "p", post)
    dv = s["dv"].double()
    du, edu = grad(dv, 0 * dv, hh, ehh, rh, pre, s["wpre"])
    dh = s["dh"].double() + du
    edh = edu + U * (dh.abs() + du.abs())
    out = {"dr": (r_scale * dh, abs(r_scale) * edh + 2 * U * dh.abs())}
    dt, edt = dh, edh
    if s["g"] is not None:
        a, sl, ea, esl = _gate(s["g"].double(), act)
        w, b = _vec(s["wpost"], 1.0, d), _vec(s["bpost"], 0.0, d)
        t = w * yh + b
        et = w.abs() * eyh + 2 * U * ((w * yh).abs() + t.abs())
        out["dg"] = (dh * t * sl, edh * (t * sl).abs() + dh.abs() * (et * sl.abs() + t.abs() * esl) + 3 * U * (dh * t * sl).abs())
        dt, edt = dh * a, edh * a.abs() + dh.abs() * ea + U * (dh * a).abs()
    out["dy"] = grad(dt, edt, yh, eyh, ry, post, s["wpost"])

    def sums(x, e):
        return x.sum(1), e.sum(1) + kn * U * x.abs().sum(1)

    out["dwpost"] = sums(dt * yh, edt * yh.abs() + dt.abs() * eyh + U * (dt * yh).abs())
    out["dbpost"] = sums(dt, edt)
    out["dwpre"] = sums(dv * hh, dv.abs() * ehh + U * (dv * hh).abs())
    out["dbpre"] = sums(dv, 0 * dv)
    return out


def _statistics(x, kind):
    x = x.double()
    m = x.mean(0) if kind == "layer" else torch.zeros_like(x[0])
    return m.float(), ((x - m).square().mean(0) + EPS).rsqrt().float()


@pytest.mark.gpu
@pytest.mark.parametrize("d,n", SHAPES)
@pytest.mark.parametrize("form", FORMS, ids=lambda f: "-".join(str(x) for x in f))
def test_backward(C, d, n, form):
    tb, ts, post, pre, act, bias, layout = form
    gen, s = _inputs(d, n, form)
    TB, TS = DT[tb], DT[ts]
    s["h"], s["dv"], s["dh"] = _mat(gen, d, n, TS, layout, 3.0), _mat(gen, d, n, TB, layout, 0.05), _mat(gen, d, n, TS, layout, 0.05)
    st = {}
    st["mp"], st["rp"] = _statistics(s["y"], post)
    st["mq"], st["rq"] = _statistics(s["h"], pre)
    ws = C.BlockNormWorkspace(d, n)
    rs = 0.9 if act != "silu" else -1.25
    want = _backward(s, post, pre, act, rs, st)

    def call(dr, accumulate, base):
        grads = {k: torch.full((d,), base, device="cuda") for k in ("dwpost", "dbpost", "dwpre", "dbpre")}
        dy, dg = _mat(gen, d, n, TB, layout), _mat(gen, d, n, TB, layout) if act is not None else None
        P = C.Norm(post, s["wpost"], s["bpost"], EPS, st["mp"], st["rp"], grads["dwpost"], grads["dbpost"])
        Q = C.Norm(pre, s["wpre"], s["bpre"], EPS, st["mq"], st["rq"], grads["dwpre"], grads["dbpre"])
        C.block_norm_bwd(s["dv"], s["dh"], s["h"], s["y"], dr, dy, ws, post=P, pre=Q, gate=s["g"], gate_act=act or "none",
                         dgate=dg, r_scale=rs, accumulate=accumulate)
        return dict(grads, dr=dr, dy=dy, dg=dg)

    first = call(_mat(gen, d, n, TS, layout), False, float("nan"))
    for name, (w, e) in want.items():
        _check(first[name], w, e, name)
    for name in ("dr", "dy", "dg"):
        if first[name] is not None:
            assert _around(first[name]).isnan().all()
    again = call(_mat(gen, d, n, TS, layout), False, float("nan"))
    for name in want:
        assert torch.equal(first[name], again[name]), name   # repeats bit for bit
    # added to what is there, over dh itself
    second = call(s["dh"], True, 2.0)
    for name in ("dr", "dy", "dg"):
        if second[name] is not None:
            assert torch.equal(first[name], second[name]), name
    for name in ("dwpost", "dbpost", "dwpre", "dbpre"):
        w, e = want[name]
        _check(second[name], 2 + w, e, name)
    assert ws.status()[0] == 0


@pytest.mark.gpu
@pytest.mark.parametrize("d,n", [(100, 40), (4096, 3), (1000, 129)])
@pytest.mark.parametrize("stream", ["bf16", "f32"])
def test_parts_left_out(C, d, n, stream):
    """Each optional part of both directions missing: the others' results are those of a neutral part in its place."""
    gen, s = _inputs(d, n, ("bf16", stream, "rms", "rms", "sigmoid", False, "tight"))
    TB, TS = DT["bf16"], DT[stream]
    e = lambda t: torch.full((d, n), float("nan"), dtype=t, device="cuda")   # noqa: E731
    w = s["wpre"]
    # the norm before the first block alone: h = r, not written
    v = e(TB)
    C.block_norm_fwd(None, s["r"], None, v, pre=C.Norm("layer", w))
    (want, err), _, _ = _norm(s["r"].double(), 2 * U * s["r"].double().abs(), "layer", w, None)
    _check(v, want, err, "v")
    # the norm after a block alone, no residual
    h = e(TS)
    C.block_norm_fwd(s["y"], None, h, None, post=C.Norm("rms", w))
    (want, err), _, _ = _norm(s["y"].double(), 0 * s["y"].double(), "rms", w, None)
    _check(h, want, err + U * want.abs(), "h")
    # a plain scaled residual
    C.block_norm_fwd(s["y"], s["r"], h, None, r_scale=0.5)
    want = 0.5 * s["r"].double() + s["y"].double()
    _check(h, want, 2 * U * (want.abs() + s["y"].double().abs()), "h")
    # no weights: those of ones
    one = torch.ones(d, device="cuda")
    v1, v2 = e(TB), e(TB)
    C.block_norm_fwd(s["y"], s["r"], h, v1, post=C.Norm("rms"), pre=C.Norm("layer"), gate=s["g"])
    C.block_norm_fwd(s["y"], s["r"], h, v2, post=C.Norm("rms", one), pre=C.Norm("layer", one, 0 * one), gate=s["g"])
    assert torch.equal(v1, v2)
    # backward
    s["h"], s["dv"], s["dh"] = _mat(gen, d, n, TS, "tight", 3.0), _mat(gen, d, n, TB), _mat(gen, d, n, TS)
    st = {}
    st["mp"], st["rp"] = _statistics(s["y"], "rms")
    st["mq"], st["rq"] = _statistics(s["h"], "rms")
    ws = C.BlockNormWorkspace(d, n)
    zero_v, zero_h = torch.zeros_like(s["dv"]), torch.zeros_like(s["dh"])

    def bwd(dv, dh, with_pre=True, with_post=True, g=s["g"], dr=True, dg=True):
        got = {k: torch.full((d,), float("nan"), device="cuda") for k in ("a", "b", "c", "d")}
        P = C.Norm("rms", w, None, EPS, None, st["rp"], got["a"], got["b"]) if with_post else None
        Q = C.Norm("rms", w, None, EPS, None, st["rq"], got["c"], got["d"]) if with_pre else None
        got.update(dr=e(TS) if dr else None, dy=e(TB), dg=e(TB) if dg else None)
        C.block_norm_bwd(dv, dh, s["h"] if with_pre else None, s["y"] if with_post or dg else None, got["dr"], got["dy"], ws,
                         post=P, pre=Q, gate=g, gate_act="silu", dgate=got["dg"], r_scale=0.9)
        return got

    def same(a, b, names):
        for k in names:
            assert torch.equal(a[k], b[k]), k

    same(bwd(None, s["dh"], with_pre=False), bwd(zero_v, s["dh"]), ("a", "b", "dr", "dy", "dg"))
    same(bwd(s["dv"], None), bwd(s["dv"], zero_h), ("a", "b", "c", "d", "dr", "dy", "dg"))
    same(bwd(s["dv"], s["dh"], dr=False, dg=False), bwd(s["dv"], s["dh"]), ("a", "b", "c", "d", "dy"))
    got = bwd(s["dv"], s["dh"], with_post=False, dg=False, g=None)
    want = _backward(dict(s, g=None, wpost=None, bpost=None, wpre=w, bpre=None), "scale", "rms", None, 0.9,
                     {"mp": None, "rp": None, "mq": None, "rq": st["rq"]})
    for k in ("dr", "dy"):
        _check(got[k], *want[k], k)
    # only the residual's part
    P = C.Norm("rms", w, None, EPS, None, st["rq"])
    dr = e(TS)
    C.block_norm_bwd(s["dv"], s["dh"], s["h"], None, dr, None, ws, pre=P, r_scale=0.9)
    _check(dr, *want["dr"], "dr alone")


@pytest.mark.gpu
@pytest.mark.parametrize("d,n", [(100, 40), (4096, 33), (1000, 1), (784, 65)])
@pytest.mark.parametrize("kind", ["rms", "layer"])
def test_hard_tokens(C, d, n, kind):
    """Columns of zeros, of one value, of a mean far above their deviation, and ones that hold NaN and infinities: every
    other token is as if they were not there."""
    gen = _gen(d + n)
    w = 1 + 0.1 * torch.randn(d, generator=gen, device="cuda")
    y = torch.randn(d, n, generator=gen, device="cuda")
    y[:, n // 2] = 0
    if n > 1:
        y[:, n // 3] = 7.25
        y[:, n - 1] = 1000 + y[:, n - 1]
        y[0, 1] = float("inf")
        y[d // 2, 0] = float("nan")
    r = torch.randn(d, n, generator=gen, device="cuda")
    bad = torch.zeros(n, dtype=torch.bool, device="cuda")
    if n > 1:
        bad[:2] = True
    h, v = torch.empty_like(y), torch.empty_like(y)
    C.block_norm_fwd(y, r, h, v, post=C.Norm(kind, w, None, EPS), pre=C.Norm(kind, w, None, EPS))
    s = {"y": y[:, ~bad], "r": r[:, ~bad], "g": None, "wpost": w, "bpost": None, "wpre": w, "bpre": None}
    (hh, eh), (vv, ev), *_ = _forward(s, kind, kind, None, 1.0)
    _check(h[:, ~bad], hh, eh, "h")
    _check(v[:, ~bad], vv, ev, "v")
    for b in bad.nonzero()[:, 0].tolist():
        assert not v[:, b].isfinite().all()
    st = {"mp": y.mean(0), "rp": torch.ones(n, device="cuda"), "mq": h.mean(0), "rq": torch.ones(n, device="cuda")}
    dy, dr = torch.empty_like(y), torch.empty_like(y)
    ws = C.BlockNormWorkspace(d, n)
    P, Q = (C.Norm(kind, w, None, EPS, st["m" + k], st["r" + k]) for k in "pq")
    C.block_norm_bwd(r, r, h, y, dr, dy, ws, post=P, pre=Q)
    s.update(dv=r[:, ~bad], dh=r[:, ~bad], h=h[:, ~bad])
    want = _backward(s, kind, kind, None, 1.0, {k: t[~bad] for k, t in st.items()})
    _check(dr[:, ~bad], *want["dr"], "dr")
    _check(dy[:, ~bad], *want["dy"], "dy")


@pytest.mark.gpu
def test_no_tokens_and_no_features(C):
    e = lambda *s: torch.empty(*s, dtype=torch.bfloat16, device="cuda")   # noqa: E731
    C.block_norm_fwd(e(16, 0), e(16, 0), e(16, 0), e(16, 0), pre=C.Norm("rms"))
    C.block_norm_fwd(e(0, 8), e(0, 8), e(0, 8), e(0, 8), pre=C.Norm("rms"))
    ws = C.BlockNormWorkspace(16, 0)
    dw, db = torch.full((16,), 3.0, device="cuda"), torch.full((16,), 3.0, device="cuda")
    rstd = torch.empty(0, device="cuda")
    for accumulate, value in ((True, 3.0), (False, 0.0)):
        C.block_norm_bwd(e(16, 0), None, e(16, 0), None, e(16, 0), None, ws, accumulate=accumulate,
                         pre=C.Norm("rms", rstd=torch.empty(1, device="cuda") if not rstd.numel() else rstd, dweight=dw, dbias=db))
        assert (dw == value).all() and (db == value).all()


@pytest.mark.gpu
def test_captured_on_another_stream(C):
    """Both directions captured together on a side stream, replayed on new inputs, beside eager calls on other buffers."""
    d, n = 520, 200
    form = ("bf16", "f32", "layer", "rms", "silu", True, "tight")
    gen, s = _inputs(d, n, form)
    h, v = torch.empty(d, n, device="cuda"), torch.empty(d, n, dtype=torch.bfloat16, device="cuda")
    st = {k: torch.empty(n, device="cuda") for k in ("mp", "rp", "mq", "rq")}
    dv, dh = _mat(gen, d, n, torch.bfloat16), _mat(gen, d, n, torch.float32)
    out = {"dr": torch.empty_like(h), "dy": torch.empty_like(v), "dg": torch.empty_like(v)}
    out.update({k: torch.empty(d, device="cuda") for k in ("a", "b", "c", "d")})
    ws = C.BlockNormWorkspace(d, n)
    P = C.Norm("layer", s["wpost"], s["bpost"], EPS, st["mp"], st["rp"], out["a"], out["b"])
    Q = C.Norm("rms", s["wpre"], s["bpre"], EPS, None, st["rq"], out["c"], out["d"])

    def run():
        C.block_norm_fwd(s["y"], s["r"], h, v, post=P, pre=Q, gate=s["g"], gate_act="silu", r_scale=0.9)
        C.block_norm_bwd(dv, dh, h, s["y"], out["dr"], out["dy"], ws, post=P, pre=Q, gate=s["g"], gate_act="silu",
                         dgate=out["dg"], r_scale=0.9)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            run()
        for seed in (1, 2):
            _, t = _inputs(d, n, form, seed)
            for k in ("y", "r", "g"):
                s[k].copy_(t[k])
            run()
            want = {k: x.clone() for k, x in dict(out, h=h, v=v).items()}
            for x in want:
                dict(out, h=h, v=v)[x].zero_()
            graph.replay()
            for k, x in dict(out, h=h, v=v).items():
                assert torch.equal(x, want[k]), k
    torch.cuda.current_stream().wait_stream(side)
    assert ws.status()[0] == 0


@pytest.mark.gpu
def test_rows_past_32_bits(C):
    """A wide buffer: the last rows begin beyond 2^31 elements."""
    d, n, ld = 600, 24, 1 << 22
    buf = torch.zeros(d * ld, dtype=torch.bfloat16, device="cuda").view(d, ld)
    gen = _gen(5)
    y, v = buf[:, 64:64 + n], buf[:, 8192:8192 + n]
    y.copy_(torch.randn(d, n, generator=gen, device="cuda"))
    w = 1 + 0.1 * torch.randn(d, generator=gen, device="cuda")
    rstd = torch.empty(n, device="cuda")
    C.block_norm_fwd(y, None, None, v, pre=C.Norm("rms", w, None, EPS, None, rstd))
    (want, err), _, _ = _norm(y.double(), U * y.double().abs(), "rms", w, None)
    _check(v, want, err, "v")
    dr = buf[:, 16384:16384 + n]
    ws = C.BlockNormWorkspace(d, n)
    C.block_norm_bwd(v, None, y, None, dr, None, ws, pre=C.Norm("rms", w, None, EPS, None, rstd))
    s = {"y": y, "h": y, "dv": v, "dh": torch.zeros_like(y), "g": None, "wpost": None, "bpost": None, "wpre": w, "bpre": None}
    _check(dr, *_backward(s, "scale", "rms", None, 1.0, {"rq": rstd, "mq": None})["dr"], "dr")


@pytest.mark.parametrize("post,pre,act", [("rms", "layer", "silu"), ("layer", "rms", "sigmoid"), ("scale", "rms", "none"),
                                          ("layer", "layer", None)])
def test_formula_against_differences(post, pre, act):
    """The formulas that the kernels are tested against, against central differences in float64 (on the CPU): third-order
    terms of a step of 1e-5 are about 1e-10, roundings 1e-16 / 1e-5."""
    gen = torch.Generator().manual_seed(3)
    d, n, rs = 7, 3, 0.9
    t = {k: torch.randn(d, n, generator=gen, dtype=torch.float64) for k in ("y", "r", "g", "cv", "ch")}
    t.update({k: 1 + 0.3 * torch.randn(d, generator=gen, dtype=torch.float64) for k in ("wpost", "bpost", "wpre", "bpre")})

    def norm(x, kind, w, b):
        if kind == "layer":
            x = x - x.mean(0)
        if kind != "scale":
            x = x / (x.square().mean(0) + EPS).sqrt()
        return x * w[:, None] + b[:, None]

    def loss(q):
        y = norm(q["y"], post, q["wpost"], q["bpost"])
        if act is not None:
            p = _sigmoid(q["g"])
            y = y * (q["g"] if act == "none" else p if act == "sigmoid" else q["g"] * p)
        h = rs * q["r"] + y
        return ((norm(h, pre, q["wpre"], q["bpre"]) * q["cv"]).sum() + (h * q["ch"]).sum()), h

    h = loss(t)[1]
    st = {}
    for side, x, kind in (("p", t["y"], post), ("q", h, pre)):
        m = x.mean(0) if kind == "layer" else torch.zeros(n, dtype=torch.float64)
        st["m" + side], st["r" + side] = m, ((x - m).square().mean(0) + EPS).rsqrt()
    s = {"y": t["y"], "h": h, "dv": t["cv"], "dh": t["ch"], "g": t["g"] if act is not None else None, "wpost": t["wpost"],
         "bpost": t["bpost"], "wpre": t["wpre"], "bpre": t["bpre"]}
    got = _backward(s, post, pre, act, rs, st)
    step = 1e-5
    for name, key in (("r", "dr"), ("y", "dy"), ("g", "dg"), ("wpost", "dwpost"), ("bpost", "dbpost"), ("wpre", "dwpre"),
                      ("bpre", "dbpre")):
        if key not in got:
            continue
        grad = got[key][0]
        for at in range(t[name].numel()):
            e = torch.zeros_like(t[name]).view(-1)
            e[at] = step
            e = e.view_as(t[name])
            num = (loss(dict(t, **{name: t[name] + e}))[0] - loss(dict(t, **{name: t[name] - e}))[0]) / (2 * step)
            assert math.isclose(float(num), float(grad.reshape(-1)[at]), rel_tol=1e-6, abs_tol=1e-7), (name, at)


@pytest.mark.gpu
@pytest.mark.parametrize("d,n,layout", [(64, 256, "tight"), (1000, 24, "wide"), (513, 33, "odd"), (70000, 1, "tight")])
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("act", ["sigmoid", "silu"])
def test_gradient_of_open_and_shut_gates(C, d, n, layout, dtype, act):
    """With dh = 1, dv = 0 and t = 1 the gate's gradient is the gate's slope: p q and p (1 + g q), q = 1 - p. Where p is
    near 1 its digits are those of e^-g. Off by, in steps of 2^-23: the exponential 2 + 1.173 |g|, two roundings of
    1 + e^-g (half a step, entering p and q), two of the reciprocal (one step each), two products (half a step each)."""
    gen, dt = _gen(d + n), DT[dtype]
    g = _mat(gen, d, n, dt, layout)
    g.copy_(torch.linspace(-80, 80, d * n, device="cuda")[torch.randperm(d * n, generator=gen, device="cuda")].view(d, n))
    y, dh, dv, h = (_mat(gen, d, n, dt, layout) for _ in range(4))
    y.fill_(1)
    dh.fill_(1)
    dv.zero_()
    dr, dy, dg = (_mat(gen, d, n, dt, layout) for _ in range(3))
    Q = C.Norm("rms", eps=EPS, rstd=_statistics(h, "rms")[1])
    ws = C.BlockNormWorkspace(d, n)
    C.block_norm_bwd(dv, dh, h, y, dr, dy, ws, post=C.Norm("scale"), pre=Q, gate=g, gate_act=act, dgate=dg)
    x = g.double()
    e = torch.exp(-x.abs())
    big, small = 1 / (1 + e), e / (1 + e)
    p, q = torch.where(x > 0, big, small), torch.where(x > 0, small, big)
    err = (6 + 1.173 * x.abs()) * 2.0 ** -23
    if act == "sigmoid":
        _check(dg, p * q, err * p * q, "slope")
    else:
        slope = p * (1 + x * q)
        _check(dg, slope, err * slope.abs() + p * (err * x.abs() * q + 2 * U * (1 + x.abs() * q)), "slope")


# A cluster walks over several tiles of tokens (a GB300 holds about 14 to 150 of them: two tiles each or more): whole vectors,
# results that end inside one, rows off the 16-byte grid, every width of the choice of tiles
LONG = [(784, 15008), (2048, 6001), (4096, 3608), (4096, 3605), (4096, 1201), (6000, 1504), (9216, 800), (12000, 401)]
LONG_FORMS = [("bf16", "bf16", "rms", "rms", "sigmoid", False, "tight"),
              ("bf16", "f32", "layer", "rms", "silu", True, "wide"),
              ("f16", "f16", "layer", "layer", "none", True, "odd"),
              ("f16", "f32", "rms", "layer", None, False, "tight"),
              ("f32", "f32", "scale", "layer", "silu", True, "tight")]


@pytest.mark.gpu
@pytest.mark.parametrize("d,n", LONG)
@pytest.mark.parametrize("form", LONG_FORMS, ids=lambda f: "-".join(str(x) for x in f))
def test_forward_over_several_tiles(C, d, n, form):
    test_forward(C, d, n, form)


@pytest.mark.gpu
@pytest.mark.parametrize("d,n", LONG)
@pytest.mark.parametrize("form", LONG_FORMS, ids=lambda f: "-".join(str(x) for x in f))
def test_backward_over_several_tiles(C, d, n, form):
    test_backward(C, d, n, form)


@pytest.mark.gpu
@pytest.mark.parametrize("d,n,layout", [(64, 256, "tight"), (1000, 24, "wide"), (513, 33, "odd"), (4096, 1, "tight"), (70000, 1, "tight")])
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("act", ["sigmoid", "silu"])
def test_infinite_gates(C, d, n, layout, dtype, act):
    """A gate that is infinite has its limits: sigmoid 0 and 1 with slopes 0, silu 0 and infinity with slopes 0 and 1. A NaN
    stays one, and the gates beside them are as if they were not there. With y = dh = 1 and no norms h is the gate's value,
    dy too, and dgate its slope."""
    gen, dt, inf = _gen(d + n), DT[dtype], float("inf")
    g = _mat(gen, d, n, dt, layout, 2.0)
    y, dh, h, dr, dy, dg = (_mat(gen, d, n, dt, layout) for _ in range(6))
    y.fill_(1)
    dh.fill_(1)
    kind = torch.randint(0, 8, (d, n), generator=gen, device="cuda")   # 0: -inf, 1: inf, 2: NaN, 3, 4: the largest finite
    top = torch.finfo(dt).max
    for k, x in enumerate((-inf, inf, float("nan"), -top, top)):
        g[kind == k] = x
    C.block_norm_fwd(y, None, h, None, post=C.Norm("scale"), gate=g, gate_act=act)
    ws = C.BlockNormWorkspace(d, n)
    C.block_norm_bwd(None, dh, None, y, dr, dy, ws, post=C.Norm("scale"), gate=g, gate_act=act, dgate=dg)
    up = (kind == 1) | (kind == 4)
    value = torch.where(up, torch.where(kind == 1, inf, top) if act == "silu" else 1.0, 0.0).to(dt)
    slope = (up if act == "silu" else up & False).to(dt)
    edge = (kind < 5) & (kind != 2)
    for got, want in ((h, value), (dy, value), (dg, slope)):
        assert (got[kind == 2].isnan()).all()
        assert (got[edge] == want[edge]).all()
    p, s, ep, es = _gate(g.double().nan_to_num(0, 0, 0), act)
    keep = kind >= 5
    for name, got, (want, err) in (("h", h, (p, ep)), ("dy", dy, (p, ep)), ("dg", dg, (s, es))):
        _check(got[keep], want[keep], err[keep] + U * want[keep].abs(), name)
    assert (dr == dh).all() and ws.status()[0] == 0


@pytest.mark.gpu
@pytest.mark.parametrize("eps", [1e-44, 1e-40, 3e-38, 1e-30, 1.0, 1e30])
@pytest.mark.parametrize("d,n", [(64, 40), (300, 1), (513, 33), (70000, 1)])
@pytest.mark.parametrize("kind", ["rms", "layer"])
def test_deviation_of_equal_features(C, d, n, kind, eps):
    """Tokens of zeros: rstd is 1 / sqrt(eps) for every eps that float32 holds (two steps of the root, two of the rest), and
    the result is the bias."""
    x = torch.zeros(d, n, device="cuda")
    rstd, v = torch.empty(n, device="cuda"), torch.full_like(x, float("nan"))
    b = torch.randn(d, generator=_gen(d), device="cuda")
    C.block_norm_fwd(None, x, None, v, pre=C.Norm(kind, None, b, eps, torch.empty(n, device="cuda"), rstd))
    want = float(torch.tensor(eps, dtype=torch.float32)) ** -0.5
    assert ((rstd.double() - want).abs() <= 4 * U * 2 * want).all()
    assert torch.equal(v, b[:, None].expand(d, n))


@pytest.fixture(scope="module")
def late(C, tmp_path_factory):
    """The binding over a build whose waits count as run out (late_waits.cu); everything else is the library's."""
    import ctypes
    import os
    import subprocess
    from paper_1905_07931_gb300 import build
    here = os.path.dirname(os.path.abspath(__file__))
    so = str(tmp_path_factory.mktemp("late") / "late_waits.so")
    r = subprocess.run([build.nvcc(), *build.ARCH, *build.NVCC_FLAGS, "-shared", "-o", so, os.path.join(here, "late_waits.cu"),
                        "-Xlinker", build.LIB, "-Xlinker", "-Bsymbolic", "-Xlinker", "-rpath=" + build.LIBDIR],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    real, over = C.lib(), ctypes.CDLL(so)
    names = ("csrt_block_norm_fwd", "csrt_block_norm_bwd")
    for name in names:
        getattr(over, name).argtypes = C._SIGS[name]

    class Lib:
        def __getattr__(self, name):
            return getattr(over if name in names else real, name)

    return Lib()


@pytest.mark.gpu
@pytest.mark.parametrize("d,n", [(300, 8000), (300, 8001), (100, 8000), (1500, 40)])
def test_results_of_waits_that_run_out(C, late, monkeypatch, d, n):
    """Waits for copies (whole vectors) and for the other blocks of a cluster (more than 128 features): what they guard is
    NaN, h and the statistics as well as v, dr as well as dy; the backward call is flagged; the next call is right."""
    form = ("bf16", "bf16", "layer", "rms", "silu", True, "tight")
    gen, s = _inputs(d, n, form)
    P = C.Norm("layer", s["wpost"], s["bpost"], EPS, *(torch.zeros(n, device="cuda") for _ in range(2)),
               *(torch.zeros(d, device="cuda") for _ in range(2)))
    Q = C.Norm("rms", s["wpre"], s["bpre"], EPS, None, torch.zeros(n, device="cuda"), *(torch.zeros(d, device="cuda") for _ in range(2)))
    h, v, dr, dy, dg = (torch.zeros_like(s["y"]) for _ in range(5))
    ws = C.BlockNormWorkspace(d, n)

    def fwd(y=s["y"], r=s["r"], v=v, post=P, pre=Q, gate=s["g"]):
        for t in (h, v, P.mean, P.rstd, Q.rstd):
            if t is not None:
                t.zero_()
        C.block_norm_fwd(y, r, h, v, post=post, pre=pre, gate=gate, gate_act="silu")

    def bwd(dv=s["y"], dh=s["r"], post=P, pre=Q):
        for t in (dr, dy, dg, P.dweight, P.dbias, Q.dweight, Q.dbias):
            t.zero_()
        ws.clear_status()
        C.block_norm_bwd(dv, dh, h, s["y"], dr, dy, ws, post=post, pre=pre, gate=s["g"], gate_act="silu", dgate=dg)

    def nan(*tensors):
        return all(bool(t.isnan().all()) for t in tensors)

    with monkeypatch.context() as m:
        m.setattr(C, "lib", lambda: late)
        fwd()
        assert nan(h, v, P.rstd, Q.rstd, P.mean)
        fwd(v=None, pre=None)
        assert nan(h, P.rstd)
        if n % 8 == 0:   # copies
            fwd(y=None, post=None, gate=None)
            assert nan(h, v, Q.rstd)
            fwd(v=None, pre=None, post=None)
            assert nan(h)
        h.copy_(s["r"])
        for t in (P.rstd, Q.rstd):
            t.fill_(1)
        P.mean.zero_()
        bwd()
        assert nan(dr, dy, dg, P.dweight, P.dbias) and ws.status()[0] == C.CSRT_DEV_TIMEOUT
        if n % 8 == 0:
            bwd(dv=None, pre=None)
            assert nan(dr, dy, dg) and ws.status()[0] == C.CSRT_DEV_TIMEOUT
    fwd()
    (hh, eh), (vv, ev), *_ = _forward(s, "layer", "rms", "silu", 1.0)
    _check(h, hh, eh, "h")
    _check(v, vv, ev, "v")
    bwd()
    assert dr.isfinite().all() and dy.isfinite().all() and ws.status()[0] == 0
