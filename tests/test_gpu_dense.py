"""Dense-layer calls against the definitions in float64.

Bounds. A product's 16-bit operands multiply exactly in float32. The tensor core adds blocks of 16 products to the
float32 accumulator with truncation (2^-23 of the running sum, itself at most S = sum |a||b|): after B = ceil(r / 16)
blocks the sum is within (B + 8) 2^-23 S. Float32 outputs are taken out every 512 terms and added rounded to nearest:
(32 + 8 + chunks) 2^-23 S. Slices of a split reduction add at most 32 more roundings. Activations have |act'| < 1.13
and are evaluated to 2^-18 of max(1, |z|); the result is rounded once to its type (2^-8 bfloat16, 2^-11 float16,
2^-24 float32, and float16's smallest step 2^-24 near zero).
"""

import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
U = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}


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
    16-byte grid)."""
    v = (torch.randn(rows, cols, generator=gen, device="cuda") * scale).to(dt)
    if layout == "tight":
        return v
    wide = (cols + 63) // 64 * 64 + 64 if layout == "wide" else cols + 5
    buf = torch.full((rows, wide), float("nan"), dtype=dt, device="cuda")
    view = buf[:, 0:cols] if layout == "wide" else buf[:, 3:3 + cols]
    view.copy_(v)
    return view


def _act(z, act):
    if act == "relu":
        return z.clamp_min(0)
    if act == "gelu":
        return 0.5 * z * (1 + torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)))
    if act == "silu":
        return z * torch.sigmoid(z)
    return z


def _act_grad(z, act):
    if act == "relu":
        return (z > 0).double()
    if act == "gelu":
        c = math.sqrt(2 / math.pi)
        t = torch.tanh(c * (z + 0.044715 * z ** 3))
        return 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * c * (1 + 3 * 0.044715 * z * z)
    if act == "silu":
        p = torch.sigmoid(z)
        return p * (1 + z * (1 - p))
    return torch.ones_like(z)


def _sum_tol(r, s, dt):
    blocks = 40 + -(-r // 512) if dt == torch.float32 else -(-r // 16) + 8
    return (blocks + 32) * 2.0 ** -23 * s


def _check(got, want, tol, dt):
    tol = tol + U[dt] * (want.abs() + tol) + (2.0 ** -24 if dt == torch.float16 else 0) + 1e-30
    bad = ~((got.double() - want).abs() <= tol)
    assert not bad.any(), (int(bad.sum()), float(((got.double() - want).abs() / tol).max()))


SIZES = [(1, 1, 1), (1, 7, 3), (5, 1, 2), (3, 9, 1), (64, 64, 4), (130, 70, 5), (200, 96, 33), (33, 700, 8), (257, 129, 63),
         (128, 64, 64), (1000, 520, 96), (256, 2048, 16), (96, 4096, 40), (2048, 72, 300), (777, 333, 511), (1024, 1024, 1024),
         (4096, 640, 700), (300, 784, 256)]


@pytest.mark.parametrize("m,k,n", SIZES)
@pytest.mark.parametrize("dtype,out,act,layout", [("bf16", None, "gelu", "tight"), ("f16", None, "silu", "odd"),
                                                  ("bf16", "f32", "relu", "wide"), ("f16", "f32", "none", "odd"),
                                                  ("bf16", None, "relu", "wide"), ("f16", None, "none", "tight")])
def test_forward(C, m, k, n, dtype, out, act, layout):
    gen, dt = _gen(m * 131 + k * 17 + n), DT[dtype]
    od = DT[out] if out else dt
    w = _mat(gen, m, k, dt, layout, 1 / math.sqrt(k))
    x = _mat(gen, k, n, dt, layout)
    b = torch.randn(m, generator=gen, device="cuda")
    r = _mat(gen, m, n, od, layout)
    y, z = _mat(gen, m, n, od, layout), _mat(gen, m, n, dt, layout)
    ws = C.DenseWorkspace(m, k, n)
    C.dense_fwd(w, x, y, ws, bias=b, act=act, residual=r, z=z)
    zz = w.double() @ x.double() + b.double()[:, None]
    s = w.double().abs() @ x.double().abs() + b.double().abs()[:, None]
    e = _sum_tol(k, s, od)
    _check(z, zz, e, dt)
    want = _act(zz, act) + r.double()
    _check(y, want, 1.13 * e + 2.0 ** -18 * zz.abs().clamp_min(1) * (act != "none") + 2.0 ** -23 * (want.abs() + r.double().abs()), od)
    # without the optional parts, and in place over the residual
    C.dense_fwd(w, x, y, ws)
    _check(y, w.double() @ x.double(), e, od)
    y2 = r.clone() if layout == "tight" else r
    want = w.double() @ x.double() + y2.double()
    C.dense_fwd(w, x, y2, ws, residual=y2)
    _check(y2, want, e + 2.0 ** -23 * want.abs(), od)
    assert ws.status()[0] == 0


@pytest.mark.parametrize("m,k,n", SIZES)
@pytest.mark.parametrize("dtype,out,act,layout", [("bf16", None, "gelu", "tight"), ("f16", None, "relu", "odd"),
                                                  ("bf16", "f32", "silu", "wide"), ("f16", None, "silu", "wide"),
                                                  ("f16", "f32", "gelu", "odd")])
def test_input_gradient(C, m, k, n, dtype, out, act, layout):
    gen, dt = _gen(m * 7 + k * 3 + n), DT[dtype]
    od = DT[out] if out else dt
    w, dy = _mat(gen, m, k, dt, layout, 1 / math.sqrt(m)), _mat(gen, m, n, dt, layout)
    z, r = _mat(gen, k, n, dt, layout), _mat(gen, k, n, od, layout)
    dx = _mat(gen, k, n, od, layout)
    ws = C.DenseWorkspace(m, k, n)
    C.dense_bwd_x(w, dy, dx, ws, z_below=z, act=act, residual=r)
    prod = w.double().t() @ dy.double()
    s = w.double().abs().t() @ dy.double().abs()
    e = _sum_tol(m, s, od)
    want = prod * _act_grad(z.double(), act) + r.double()
    tol = 1.13 * e + 2.0 ** -17 * prod.abs() * z.double().abs().clamp_min(1) + 2.0 ** -23 * (want.abs() + r.double().abs())
    _check(dx, want, tol, od)
    C.dense_bwd_x(w, dy, dx, ws)
    _check(dx, prod, e, od)
    assert ws.status()[0] == 0


@pytest.mark.parametrize("m,k,n", SIZES + [(70, 90, 5000), (8192, 64, 2048)])
@pytest.mark.parametrize("dtype,out,layout", [("bf16", "f32", "tight"), ("f16", "f32", "odd"), ("bf16", None, "wide"),
                                              ("f16", None, "odd")])
def test_weight_gradient(C, m, k, n, dtype, out, layout):
    gen, dt = _gen(m + k + n), DT[dtype]
    od = DT[out] if out else dt
    dy, x = _mat(gen, m, n, dt, layout), _mat(gen, k, n, dt, layout)
    dw, db = _mat(gen, m, k, od, layout), torch.zeros(m, device="cuda")
    ws = C.DenseWorkspace(m, k, n)
    C.dense_bwd_w(dy, x, dw, ws, db=db)
    want, s = dy.double() @ x.double().t(), dy.double().abs() @ x.double().abs().t()
    e = _sum_tol(n, s, od)
    _check(dw, want, e, od)
    sb = dy.double().abs().sum(1)
    _check(db, dy.double().sum(1), (n / 32 + 16) * 2.0 ** -23 * sb, torch.float32)
    before = dw.double().clone()
    db0 = db.clone()
    C.dense_bwd_w(dy, x, dw, ws, db=db, accumulate=True)
    _check(dw, want + before, e + 2.0 ** -22 * (want.abs() + before.abs()), od)
    _check(db, db0.double() * 2, (n / 32 + 17) * 2.0 ** -23 * 2 * sb, torch.float32)
    assert ws.status()[0] == 0


@pytest.mark.parametrize("act", ["relu", "gelu", "silu"])
def test_gradients_against_differences(C, act):
    """d/dt of f = sum(c * y) along a direction of x, W and b equals the calls' gradients contracted with it."""
    gen, m, k, n = _gen(5), 40, 56, 24
    w = (_mat(gen, m, k, torch.float32) / math.sqrt(k)).to(torch.float16)
    x, c = _mat(gen, k, n, torch.float16), _mat(gen, m, n, torch.float16)
    b = torch.randn(m, generator=gen, device="cuda")
    ws = C.DenseWorkspace(m, k, n)
    y, z = torch.empty(m, n, device="cuda"), torch.empty(m, n, dtype=torch.float16, device="cuda")
    C.dense_fwd(w, x, y, ws, bias=b, act=act, z=z)
    dpre = torch.empty(m, n, dtype=torch.float16, device="cuda")
    C.dense_act_bwd(c, z, act, dpre)
    dx, dw, db = torch.empty(k, n, device="cuda"), torch.empty(m, k, device="cuda"), torch.empty(m, device="cuda")
    C.dense_bwd_x(w, dpre, dx, ws)
    C.dense_bwd_w(dpre, x, dw, ws, db=db)

    def f(dwt, dxt, dbt, t):
        zz = (w.double() + t * dwt) @ (x.double() + t * dxt) + (b.double() + t * dbt)[:, None]
        return (c.double() * _act(zz, act)).sum()

    zero = (torch.zeros(m, k, device="cuda").double(), torch.zeros(k, n, device="cuda").double(),
            torch.zeros(m, device="cuda").double())
    for i, g in enumerate((dw, dx, db)):
        for s in range(3):
            d = torch.randn(g.shape, generator=_gen(100 + 10 * i + s), device="cuda").double()
            args = list(zero)
            args[i] = d
            h = 1e-5
            num = float((f(*args, h) - f(*args, -h)) / (2 * h))
            ana = float((g.double() * d).sum())
            # dpre, z and the kink of relu: 2^-11 relative per rounding, summed in quadrature over the entries
            scale = float((g.double().abs() * d.abs()).sum())
            assert abs(num - ana) <= 2e-2 * scale / math.sqrt(g.numel()) * 4 + 1e-6, (i, s, num, ana, scale)


@pytest.mark.parametrize("rows,cols", [(1, 1), (3, 1000), (257, 33), (1024, 513)])
@pytest.mark.parametrize("act", ["none", "relu", "gelu", "silu"])
@pytest.mark.parametrize("din,dz,dout", [("bf16", "bf16", "bf16"), ("f32", "f16", "f16"), ("f16", "f32", "f32")])
def test_act_bwd(C, rows, cols, act, din, dz, dout):
    gen = _gen(rows + cols)
    dy, z = _mat(gen, rows, cols, DT[din], "odd"), _mat(gen, rows, cols, DT[dz], "wide")
    out = _mat(gen, rows, cols, DT[dout], "odd")
    C.dense_act_bwd(dy, z, act, out)
    want = dy.double() * _act_grad(z.double(), act)
    _check(out, want, 2.0 ** -17 * dy.double().abs() * z.double().abs().clamp_min(1) * (act != "none") + 2.0 ** -23 * want.abs(), DT[dout])
    if din == dout:   # in place
        C.dense_act_bwd(dy, z, act, dy)
        assert torch.equal(dy, out)


def test_dense_update_is_exact(C):
    gen = _gen(9)
    w, d = _mat(gen, 70, 130, torch.float32), _mat(gen, 70, 130, torch.bfloat16, "odd")
    w16 = _mat(gen, 70, 130, torch.float16, "wide")
    eta, decay = 0.03, 0.1
    keep = (1.0 - torch.tensor(eta, dtype=torch.float32) * torch.tensor(decay, dtype=torch.float32)).float().cuda()
    want = w * keep - torch.tensor(eta, dtype=torch.float32, device="cuda") * d.float()
    C.dense_update(w, d, eta, decay, w16)
    assert torch.equal(w, want) and torch.equal(w16, want.to(torch.float16))


def test_empty_reductions_and_empty_outputs(C):
    b = torch.randn(6, device="cuda")
    ws = C.DenseWorkspace(64, 64, 64)
    for n in (3, 40):   # both forward paths
        w, x = torch.empty(6, 0, dtype=torch.bfloat16, device="cuda"), torch.empty(0, n, dtype=torch.bfloat16, device="cuda")
        y = torch.full((6, n), float("nan"), dtype=torch.bfloat16, device="cuda")
        C.dense_fwd(w, x, y, ws, bias=b, act="relu")
        assert torch.equal(y, b.clamp_min(0).to(torch.bfloat16)[:, None].expand(6, n))
    dy, x = torch.empty(6, 0, dtype=torch.float16, device="cuda"), torch.empty(9, 0, dtype=torch.float16, device="cuda")
    dw, db = torch.ones(6, 9, device="cuda"), torch.ones(6, device="cuda")
    C.dense_bwd_w(dy, x, dw, ws, db=db, accumulate=True)
    assert bool((dw == 1).all()) and bool((db == 1).all())
    C.dense_bwd_w(dy, x, dw, ws, db=db)
    assert bool((dw == 0).all()) and bool((db == 0).all())


def test_infinities_and_nans_stay_in_their_rows_and_columns(C):
    gen = _gen(3)
    m, k, n = 200, 150, 90
    w, x = _mat(gen, m, k, torch.bfloat16), _mat(gen, k, n, torch.bfloat16).abs() + 0.5
    w[17, 3] = float("inf")
    w[60, 5] = float("nan")
    y = torch.empty(m, n, dtype=torch.bfloat16, device="cuda")
    ws = C.DenseWorkspace(m, k, n)
    C.dense_fwd(w, x, y, ws, act="silu")
    assert bool((y[17] == float("inf")).all()) and bool(y[60].isnan().all())
    rest = [i for i in range(m) if i not in (17, 60)]
    assert bool(y[rest].isfinite().all())


@pytest.mark.parametrize("n", [1, 4, 24, 200])
def test_results_repeat_bit_for_bit(C, n):
    gen = _gen(n)
    m, k = 600, 5000
    w, x = _mat(gen, m, k, torch.bfloat16), _mat(gen, k, n, torch.bfloat16)
    ws, outs = C.DenseWorkspace(m, k, n), []
    for _ in range(4):
        y, dx = torch.empty(m, n, device="cuda"), torch.empty(k, n, dtype=torch.bfloat16, device="cuda")
        dw, db = torch.empty(m, k, device="cuda"), torch.empty(m, device="cuda")
        C.dense_fwd(w, x, y, ws)
        dy = y.to(torch.bfloat16)
        C.dense_bwd_x(w, dy, dx, ws)
        C.dense_bwd_w(dy, x, dw, ws, db=db)
        outs.append((y, dx, dw, db))
    for o in outs[1:]:
        assert all(torch.equal(a, b) for a, b in zip(o, outs[0]))


def test_offsets_beyond_32_bits(C):
    """Rows 2^26 elements apart: the last ones lie past 2^32 elements."""
    gen, k, m, n, ld = _gen(4), 72, 66, 40, 1 << 26
    buf = torch.empty(k, ld, dtype=torch.bfloat16, device="cuda")
    out = torch.empty(m, ld, dtype=torch.bfloat16, device="cuda")
    x, y = buf[:, 64:64 + n], out[:, 128:128 + n]
    x.copy_(torch.randn(k, n, generator=gen, device="cuda"))
    w = _mat(gen, m, k, torch.bfloat16)
    ws = C.DenseWorkspace(m, k, n)
    for xx, yy in ((x, y), (x[:, :3], y[:, 1:4])):   # tensor cores; few tokens, off the 16-byte grid
        C.dense_fwd(w, xx, yy, ws, residual=None)
        want, s = w.double() @ xx.double(), w.double().abs() @ xx.double().abs()
        _check(yy, want, _sum_tol(k, s, torch.bfloat16), torch.bfloat16)
    del buf, out
    torch.cuda.empty_cache()


def test_calls_run_on_the_given_stream_and_in_a_graph(C):
    gen, m, k, n = _gen(8), 256, 512, 96
    w, x = _mat(gen, m, k, torch.bfloat16), _mat(gen, k, n, torch.bfloat16)
    y = torch.zeros(m, n, dtype=torch.bfloat16, device="cuda")
    want = torch.empty_like(y)
    ws = C.DenseWorkspace(m, k, n)
    C.dense_fwd(w, x, want, ws)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        torch.cuda._sleep(20_000_000)
        x2 = x * 2
    C.dense_fwd(w, x2, y, ws, stream=s)   # after the sleep and the product on s
    s.synchronize()
    assert torch.equal(y, (want.float() * 2).to(torch.bfloat16))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        C.dense_fwd(w, x, y, ws)
    y.zero_()
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(y, want)


def test_binding_refuses(C):
    w = torch.zeros(8, 16, dtype=torch.bfloat16, device="cuda")
    x, y = torch.zeros(16, 4, dtype=torch.bfloat16, device="cuda"), torch.zeros(8, 4, dtype=torch.bfloat16, device="cuda")
    ws = C.DenseWorkspace(8, 16, 4)
    with pytest.raises(ValueError, match="contiguous"):
        C.dense_fwd(w, x.t().contiguous().t(), y, ws)
    with pytest.raises(ValueError, match="2-D"):
        C.dense_fwd(w, x[0], y, ws)
    with pytest.raises(ValueError, match="not supported"):
        C.dense_fwd(w.double(), x, y, ws)
    with pytest.raises(ValueError, match="unknown activation"):
        C.dense_fwd(w, x, y, ws, act="tanh")
    with pytest.raises(C.CsrtError, match="must be 16 x 4"):
        C.dense_fwd(w, x[:15], y, ws)
    with pytest.raises(ValueError, match="bias"):
        C.dense_fwd(w, x, y, ws, bias=torch.zeros(4, device="cuda"))
    with pytest.raises(C.CsrtError, match="workspace has"):
        C.dense_fwd(torch.zeros(4096, 16, dtype=torch.bfloat16, device="cuda"), x,
                    torch.zeros(4096, 4, dtype=torch.bfloat16, device="cuda"), ws)


@pytest.mark.parametrize("m,k,n", [(96, 72, 40), (70, 40, 3), (130, 33, 1), (200, 160, 136)])
@pytest.mark.parametrize("odd", [0, 3])
def test_rows_far_apart(C, m, k, n, odd):
    """Matrices whose last row lies past 2^31 elements give the bits of the same rows close together."""
    gen = _gen(m + k + n + odd)
    bufs = []

    def pair(rows, cols, dt):
        close = (cols + 63) // 64 * 64 + odd
        far = (2 ** 31 // (rows - 1) // 64 + 1) * 64 + odd
        out = []
        v = torch.randn(rows, cols, generator=gen, device="cuda").to(dt)
        for ld in (close, far):
            buf = torch.empty(odd + (rows - 1) * ld + cols, dtype=dt, device="cuda")
            bufs.append(buf)
            out.append(buf.as_strided((rows, cols), (ld, 1), odd))
            out[-1].copy_(v)
        return out

    ws = C.DenseWorkspace(m, k, n)
    bias = torch.randn(m, generator=gen, device="cuda")
    bf, f32 = torch.bfloat16, torch.float32
    w, x, r, z, y = pair(m, k, bf), pair(k, n, bf), pair(m, n, bf), pair(m, n, bf), pair(m, n, bf)
    for i in range(2):
        C.dense_fwd(w[i], x[i], y[i], ws, bias=bias, act="gelu", residual=r[i], z=z[i])
    assert torch.equal(y[0], y[1]) and torch.equal(z[0], z[1])
    del r
    bufs.clear()
    dx, dw, zb = pair(k, n, bf), pair(m, k, f32), pair(k, n, bf)
    db = torch.zeros(2, m, device="cuda")
    for i in range(2):
        C.dense_bwd_x(w[i], z[i], dx[i], ws, z_below=zb[i], act="silu")
        C.dense_bwd_w(z[i], x[i], dw[i], ws, db=db[i], accumulate=True)
    assert torch.equal(dx[0], dx[1]) and torch.equal(dw[0], dw[1]) and torch.equal(db[0], db[1])
    w16 = pair(m, k, bf)
    for i in range(2):
        C.dense_update(dw[i], w[i], 0.1, 0.01, w16[i])
        C.dense_act_bwd(z[i], x[i] if m == k else z[i], "gelu", y[i])
    assert torch.equal(dw[0], dw[1]) and torch.equal(w16[0], w16[1]) and torch.equal(y[0], y[1])


@pytest.mark.parametrize("act", ["gelu", "silu"])
@pytest.mark.parametrize("dtype,n", [("bf16", 16), ("bf16", 13), ("f16", 16), ("f16", 13)])
def test_derivatives_far_from_zero(C, act, dtype, n):
    """act' is 1 (z > 0) or 0 (z < 0) within float32 where |z| is large, up to infinities: those that float16 keeps of a
    pre-activation beyond 65504, and bfloat16's whole range."""
    dt, inf = DT[dtype], float("inf")
    big = [120.0, 6e4, inf] + ([1e13, 1e19, 1e25, 3e38] if dtype == "bf16" else [200.0])
    z = torch.tensor(big + [-v for v in big], device="cuda").to(dt)
    k, m = z.numel(), 40
    one = (z > 0).to(dt)
    zz = z[:, None].repeat(1, n).contiguous()
    dy = _mat(_gen(n), k, n, dt)
    out = torch.empty_like(dy)
    C.dense_act_bwd(dy, zz, act, out)
    assert torch.equal(out, dy * one[:, None])
    # the same in the epilogue of the input gradient: the plain product where z > 0, nothing elsewhere
    w, g = _mat(_gen(1), m, k, dt), _mat(_gen(2), m, n, dt)
    dx, plain = torch.empty(k, n, dtype=dt, device="cuda"), torch.empty(k, n, dtype=dt, device="cuda")
    ws = C.DenseWorkspace(m, k, n)
    C.dense_bwd_x(w, g, plain, ws)
    C.dense_bwd_x(w, g, dx, ws, z_below=zz, act=act)
    assert torch.equal(dx, plain * one[:, None])
    # a NaN is not taken for a large number
    zz[0] = float("nan")
    C.dense_act_bwd(dy, zz, act, out)
    assert bool(out[0].isnan().all()) and not bool(out[1:].isnan().any())


@pytest.mark.parametrize("kind,m,k,n,dtype,odd", [
    ("dw", 2048, 2048, 300000, "f16", 0),     # whole sums
    ("dw", 2000, 2001, 300000, "f16", 1),     # the same at odd rows
    ("dw", 2048, 2048, 40000, "f16", 0),      # just above what float16 takes in one go
    ("dw", 1000, 1000, 400000, "f16", 0),     # long slices
    ("dw", 64, 60, 2000000, "f16", 0),        # one tile in as many slices as there are
    ("dw", 2048, 2048, 1200000, "bf16", 0),
    ("fwd", 2048, 300000, 2048, "f16", 0),
    ("fwd", 2040, 300000, 2049, "f16", 1),
    ("dx", 300000, 2048, 2048, "f16", 0),
    ("dx", 300000, 2001, 2000, "f16", 1)])
def test_long_sums_of_one_sign_are_rounded_once(C, kind, m, k, n, dtype, odd):
    """16-bit results of long reductions. Up to 32768 (float16) or 131072 (bfloat16) terms lose at most 2^-23 of the
    running sum with each block of 16; longer ones are float32 sums of 512 terms each, rounded to nearest (32 + chunks).
    Then up to 32 slices, and the result's own rounding."""
    gen, dt = _gen(m + k + n), DT[dtype]
    lay = "odd" if odd else "tight"

    def positive(rows, cols, f):
        v = torch.rand(rows, cols, generator=gen, device="cuda", dtype=torch.float32).mul_(0.1 * f).add_(0.05 * f).to(dt)
        if not odd:
            return v
        buf = torch.zeros(rows, cols + 5, dtype=dt, device="cuda")
        buf[:, 3:3 + cols].copy_(v)
        return buf[:, 3:3 + cols]

    r = {"dw": n, "fwd": k, "dx": m}[kind]
    f = min(1.0, math.sqrt(2e5 / r))       # within float16's range
    ws = C.DenseWorkspace(m, k, n)
    if kind == "dw":
        a, b, out = positive(m, n, f), positive(k, n, f), _mat(gen, m, k, dt, lay)
        C.dense_bwd_w(a, b, out, ws)
        want = a[:64].double() @ b[:64].double().t()
        far = a[-32:].double() @ b[-32:].double().t()
    elif kind == "fwd":
        a, b, out = positive(m, k, f), positive(k, n, f), _mat(gen, m, n, dt, lay)
        C.dense_fwd(a, b, out, ws)
        want, far = a[:64].double() @ b[:, :64].double(), a[-32:].double() @ b[:, -32:].double()
    else:
        a, b, out = positive(m, k, f), positive(m, n, f), _mat(gen, k, n, dt, lay)
        C.dense_bwd_x(a, b, out, ws)
        want, far = a[:, :64].double().t() @ b[:, :64].double(), a[:, -32:].double().t() @ b[:, -32:].double()
    limit = 32768 if dtype == "f16" else 131072
    tol = (max(min(r, limit) // 16, 32 + r // 512) + 32) * 2.0 ** -23
    for got, exact in ((out[:64, :64], want), (out[-32:, -32:], far)):
        exact = exact[:got.shape[0], :got.shape[1]]
        assert float(exact.max()) < 6e4
        _check(got, exact, tol * exact, dt)
    assert ws.status()[0] == 0


@pytest.mark.parametrize("kind,m,k,n", [("fwd", 200, 20000, 130), ("fwd", 2030, 70000, 2050), ("dx", 70000, 2000, 2001)])
@pytest.mark.parametrize("layout", ["tight", "odd"])
def test_long_sums_with_every_epilogue(C, kind, m, k, n, layout):
    gen, dt = _gen(m + n), torch.float16
    ws = C.DenseWorkspace(m, k, n)
    w = _mat(gen, m, k, dt, layout, 1 / math.sqrt(k if kind == "fwd" else m))
    if kind == "fwd":
        x, b, r = _mat(gen, k, n, dt, layout), torch.randn(m, generator=gen, device="cuda"), _mat(gen, m, n, dt, layout)
        y, z = _mat(gen, m, n, dt, layout), _mat(gen, m, n, dt, layout)
        C.dense_fwd(w, x, y, ws, bias=b, act="silu", residual=r, z=z)
        zz, s = w.double() @ x.double() + b.double()[:, None], w.double().abs() @ x.double().abs()
        e = _sum_tol(min(k, 32768), s, dt)
        _check(z, zz, e, dt)
        want = _act(zz, "silu") + r.double()
        _check(y, want, 1.13 * e + 2.0 ** -18 * zz.abs().clamp_min(1) + 2.0 ** -23 * (want.abs() + r.double().abs()), dt)
    else:
        dy, z, r = _mat(gen, m, n, dt, layout), _mat(gen, k, n, dt, layout), _mat(gen, k, n, dt, layout)
        dx = _mat(gen, k, n, dt, layout)
        C.dense_bwd_x(w, dy, dx, ws, z_below=z, act="gelu", residual=r)
        prod, s = w.double().t() @ dy.double(), w.double().abs().t() @ dy.double().abs()
        e = _sum_tol(min(m, 32768), s, dt)
        want = prod * _act_grad(z.double(), "gelu") + r.double()
        _check(dx, want, 1.13 * e + 2.0 ** -17 * prod.abs() * z.double().abs().clamp_min(1) +
               2.0 ** -23 * (want.abs() + r.double().abs()), dt)
    assert ws.status()[0] == 0


def _marked(rows, cols, at):
    """bfloat16 zeros with powers of two at the given places, so that every order of a sum is exact."""
    t = torch.zeros(rows, cols, dtype=torch.bfloat16, device="cuda")
    for i, (r, c) in enumerate(at):
        t[r, c] = 2.0 ** (i % 8)
    return t


@pytest.mark.parametrize("n", [2 ** 31 - 1, 2 ** 31 - 8])
@pytest.mark.parametrize("k", [0, 1])
def test_bias_gradient_of_rows_near_2_31_columns(C, n, k):
    """The last steps of a row's sum pass 2^31; with the product's idle warps (k = 1) and by itself."""
    at = [(0, 0), (0, 2 ** 30), (0, 2 ** 31 - 300), (0, 2 ** 31 - 40), (0, n - 9), (0, n - 1)]
    dy, x = _marked(1, n, at), torch.ones(k, n, dtype=torch.bfloat16, device="cuda")
    dw, db, ws = torch.zeros(1, k, device="cuda"), torch.zeros(1, device="cuda"), C.DenseWorkspace(1, k, n)
    C.dense_bwd_w(dy, x, dw, ws, db=db)
    assert float(db) == 63.0 and bool((dw == 63.0).all())
    assert ws.status()[0] == 0
    del dy, x, ws
    torch.cuda.empty_cache()


def test_bias_gradient_near_2_31_rows(C):
    m = 2 ** 31 - 100
    rows = [0, 2 ** 30 + 1, m - 305, m - 204, m - 1]
    dy, x = _marked(m, 1, [(r, 0) for r in rows]), torch.ones(1, 1, dtype=torch.bfloat16, device="cuda")
    dw, db, ws = torch.empty(m, 1, device="cuda"), torch.empty(m, device="cuda"), C.DenseWorkspace(m, 1, 1)
    C.dense_bwd_w(dy, x, dw, ws, db=db)
    for got in (dw.view(-1), db):
        assert [float(got[r]) for r in rows] == [1.0, 2.0, 4.0, 8.0, 16.0]
        assert int(torch.count_nonzero(got)) == 5 and float(got.sum()) == 31.0
    assert ws.status()[0] == 0
    del dy, dw, db, ws, got
    torch.cuda.empty_cache()


def test_one_token_of_nearly_2_31_inputs(C):
    k = 2 ** 31 - 9      # no multiple of eight: a lane's last steps pass 2^31
    w = _marked(2, k, [(0, 0), (1, 1), (0, 2 ** 31 - 300), (1, 2 ** 31 - 40), (0, k - 2), (1, k - 1)])
    x, y = torch.ones(k, 1, dtype=torch.bfloat16, device="cuda"), torch.zeros(2, 1, device="cuda")
    ws = C.DenseWorkspace(2, k, 1)
    C.dense_fwd(w, x, y, ws)
    assert y.view(-1).tolist() == [1.0 + 4 + 16, 2.0 + 8 + 32]
    assert ws.status()[0] == 0
    del w, x, ws
    torch.cuda.empty_cache()


def test_nearly_2_31_columns(C):
    """One row of 2^31 - 1 columns through the epilogues: a float32 residual of aligned rows, z and bias at odd ones."""
    n = 2 ** 31 - 1
    at = torch.tensor([0, 1, 2 ** 30, n - 32, n - 4, n - 1], device="cuda")
    vals = torch.tensor([1.0, -2.0, 3.0, -4.0, 5.0, 6.0], device="cuda")
    x = torch.zeros(1, n, dtype=torch.bfloat16, device="cuda")
    x[0, at] = vals.bfloat16()
    r = torch.empty(1, n + 1, device="cuda")[:, :n]
    r.fill_(0.5)
    w, b = torch.full((1, 1), 2.0, dtype=torch.bfloat16, device="cuda"), torch.ones(1, device="cuda")
    y, ws = torch.empty(1, n, device="cuda"), C.DenseWorkspace(1, 1, n)
    C.dense_fwd(w, x, y, ws, bias=b, residual=r.as_strided((1, n), (n + 1, 1)))
    assert torch.equal(y[0, at], 2 * vals + 1.5) and int((y == 1.5).sum()) == n - 6
    z = torch.ones(1, n, dtype=torch.bfloat16, device="cuda")
    z[0, at[1]] = -1.0
    C.dense_bwd_x(w, x, y, ws, z_below=z, act="relu", residual=r.as_strided((1, n), (n + 1, 1)))
    want = 2 * vals + 0.5
    want[1] = 0.5
    assert torch.equal(y[0, at], want) and int((y == 0.5).sum()) == n - 5
    assert ws.status()[0] == 0
    del x, r, y, z, ws
    torch.cuda.empty_cache()


@pytest.mark.parametrize("m,k,n", [(512, 640, 777), (1000, 520, 1777), (4096, 1024, 1025)])
@pytest.mark.parametrize("accumulate", [False, True])
def test_bias_gradient_of_unaligned_rows_is_the_aligned_ones(C, m, k, n, accumulate):
    """The row sums that go along with a product are taken of aligned rows in either case, in one order."""
    gen, ws, res = _gen(m + n), C.DenseWorkspace(m, k, n), []
    v, x = _mat(gen, m, n, torch.bfloat16), _mat(gen, k, n, torch.bfloat16)
    for off, wide in ((0, (n + 63) // 64 * 64), (3, n + 6)):
        buf = torch.full((m, wide), float("nan"), dtype=torch.bfloat16, device="cuda")
        dy = buf[:, off:off + n]
        dy.copy_(v)
        dw, db = torch.ones(m, k, device="cuda"), torch.ones(m, device="cuda")
        C.dense_bwd_w(dy, x, dw, ws, db=db, accumulate=accumulate)
        res.append((dw, db))
    assert torch.equal(res[0][0], res[1][0]) and torch.equal(res[0][1], res[1][1])
    want = v.double().sum(1) + accumulate
    _check(res[1][1], want, (n / 32 + 17) * 2.0 ** -23 * (v.double().abs().sum(1) + 1), torch.float32)


@pytest.mark.parametrize("n", [1, 3, 4, 5, 7, 8, 9, 12, 30, 33, 100, 130, 257, 516])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("wide", [False, True])
def test_nothing_is_written_between_rows(C, n, dtype, wide):
    """Outputs that are the first columns of aligned wider rows: the other columns, and what follows, stay as they are."""
    gen, dt, m, k = _gen(n), DT[dtype], 150, 72
    od, ld = torch.float32 if wide else dt, (n + 63) // 64 * 64 + 64

    def out(rows, cols, t, skip=0):
        buf = torch.full((rows + 1, ld), 7.0, dtype=t, device="cuda")
        return buf, buf[:rows, skip:skip + cols]

    def untouched(buf, view, skip=0):
        rest = torch.ones_like(buf, dtype=torch.bool)
        rest[:view.shape[0], skip:skip + view.shape[1]] = False
        assert bool((buf[rest] == 7.0).all())

    w, x, dy = _mat(gen, m, k, dt, "tight", 0.1), _mat(gen, k, n, dt), _mat(gen, m, n, dt, "tight", 0.1)
    ws = C.DenseWorkspace(m, k, n)
    for skip in (0, 16):
        (yb, y), (zb, z) = out(m, n, od, skip), out(m, n, dt, skip)
        C.dense_fwd(w, x, y, ws, act="gelu", z=z)
        untouched(yb, y, skip), untouched(zb, z, skip)
        zz = w.double() @ x.double()
        e = _sum_tol(k, w.double().abs() @ x.double().abs(), od)
        _check(z, zz, e, dt)
        yb, y = out(m, n, od, skip)
        C.dense_fwd(w, x, y, ws)
        untouched(yb, y, skip)
        _check(y, zz, e, od)
        xb, dx = out(k, n, od, skip)
        C.dense_bwd_x(w, dy, dx, ws)
        untouched(xb, dx, skip)
        _check(dx, w.double().t() @ dy.double(), _sum_tol(m, w.double().abs().t() @ dy.double().abs(), od), od)
        a, b = _mat(gen, m, k, dt), _mat(gen, n, k, dt)
        wb, dw = out(m, n, od, skip)
        C.dense_bwd_w(a, b, dw, C.DenseWorkspace(m, n, k))
        untouched(wb, dw, skip)
        _check(dw, a.double() @ b.double().t(), _sum_tol(k, a.double().abs() @ b.double().abs().t(), od), od)
        pb, pre = out(m, n, od, skip)
        C.dense_act_bwd(dy, dy, "silu", pre)
        untouched(pb, pre, skip)
    assert ws.status()[0] == 0


@pytest.mark.parametrize("m,k", [(300, 784), (1000, 2048), (4096, 4096), (4096, 4097), (2050, 5000)])
@pytest.mark.parametrize("n", [1, 2, 3, 4])
@pytest.mark.parametrize("ld,off", [(64, 0), (64, 5), (61, 2), (8, 1)])
def test_tokens_that_are_columns_of_a_wider_buffer(C, m, k, n, ld, off):
    """A few columns of x, z and y between others, which stay as they are: small products and large ones."""
    gen, dt = _gen(m + k + n + ld), torch.bfloat16
    w, b = _mat(gen, m, k, dt, "tight", 1 / math.sqrt(k)), torch.randn(m, generator=gen, device="cuda")
    xb = torch.randn(k, ld, generator=gen, device="cuda").to(dt)
    yb = torch.full((m, ld), 7.0, dtype=dt, device="cuda")
    zb = yb.clone()
    x, y, z = xb[:, off:off + n], yb[:, off:off + n], zb[:, off:off + n]
    ws = C.DenseWorkspace(m, k, n)
    C.dense_fwd(w, x, y, ws, bias=b, act="gelu", z=z)
    zz = w.double() @ x.double() + b.double()[:, None]
    s = w.double().abs() @ x.double().abs() + b.double().abs()[:, None]
    e = _sum_tol(k, s, dt)
    _check(z, zz, e, dt)
    _check(y, _act(zz, "gelu"), 1.13 * e + 2.0 ** -18 * zz.abs().clamp_min(1), dt)
    for buf in (yb, zb):
        assert bool((buf[:, :off] == 7).all()) and bool((buf[:, off + n:] == 7).all())
    assert ws.status()[0] == 0


# Rows, columns and reduction of products that the launcher puts on each of its tiles (256 x 256 and 256 x 128 by pairs of
# SMs, 128 x 128, 128 x 64) with whole reductions, with all tiles in slices and with the left-over ones in slices.
ON_EVERY_TILE = [(647, 3256, 72), (682, 5064, 64), (180, 4944, 6560), (5936, 216, 8464), (3170, 1584, 3016), (1193, 4048, 4200),
                 (157, 5056, 64), (148, 4880, 64), (64, 5216, 4016), (136, 2560, 4872), (522, 4384, 8064), (70, 96, 64),
                 (70, 64, 3176), (154, 4880, 1320), (154, 5072, 2976), (141, 1824, 5496), (5097, 72, 8632), (677, 3224, 6984),
                 (395, 5632, 6952)]
ON_EVERY_TILE_ODD = [(1034, 3315, 64), (202, 5233, 8496), (2737, 1859, 4040), (133, 4971, 104), (73, 5105, 4880),
                     (522, 4383, 8064), (153, 5523, 2648), (5779, 65, 8296), (2792, 841, 6784), (80, 77, 3200), (70, 65, 64)]


@pytest.mark.parametrize("rows,cols,r", ON_EVERY_TILE + ON_EVERY_TILE_ODD)
@pytest.mark.parametrize("op", ["fwd", "dx", "dw"])
@pytest.mark.parametrize("dtype,out", [("f16", None), ("bf16", "f32")])
def test_every_tile_with_every_epilogue(C, rows, cols, r, op, dtype, out):
    gen, dt = _gen(rows + cols + r), DT[dtype]
    od = DT[out] if out else dt
    base = _mat(gen, rows, cols, od)       # residual, or what is there
    there = base.double()
    ws = C.DenseWorkspace(*{"fwd": (rows, r, cols), "dx": (r, rows, cols), "dw": (rows, cols, r)}[op])
    o1, o2 = torch.empty(rows, cols, dtype=od, device="cuda"), torch.empty(rows, cols, dtype=od, device="cuda")
    s = 1 / math.sqrt(r)
    if op == "fwd":
        a, b = _mat(gen, rows, r, dt, scale=s), _mat(gen, r, cols, dt)
        prod, mag = a.double() @ b.double(), a.double().abs() @ b.double().abs()
        bias, z = torch.randn(rows, generator=gen, device="cuda"), torch.empty(rows, cols, dtype=dt, device="cuda")
        C.dense_fwd(a, b, o1, ws)
        C.dense_fwd(a, b, o2, ws, bias=bias, act="silu", residual=base, z=z)
        e = _sum_tol(r, mag, od)
        zz = prod + bias.double()[:, None]
        _check(z, zz, e + 2.0 ** -23 * zz.abs(), dt)
        want = _act(zz, "silu") + there
        tol = 1.13 * e + 2.0 ** -18 * zz.abs().clamp_min(1) + 2.0 ** -23 * (want.abs() + there.abs())
        _check(o2, want, tol, od)
        C.dense_fwd(a, b, base, ws, residual=base)     # in place
        _check(base, prod + there, e + 2.0 ** -23 * (prod + there).abs(), od)
    elif op == "dx":
        a, b = _mat(gen, r, rows, dt, scale=s), _mat(gen, r, cols, dt)
        prod, mag = a.double().t() @ b.double(), a.double().abs().t() @ b.double().abs()
        z = _mat(gen, rows, cols, dt)
        C.dense_bwd_x(a, b, o1, ws)
        C.dense_bwd_x(a, b, o2, ws, z_below=z, act="gelu", residual=base)
        e = _sum_tol(r, mag, od)
        want = prod * _act_grad(z.double(), "gelu") + there
        tol = 1.13 * e + 2.0 ** -17 * prod.abs() * z.double().abs().clamp_min(1)
        _check(o2, want, tol + 2.0 ** -23 * (want.abs() + there.abs()), od)
        C.dense_bwd_x(a, b, base, ws, z_below=z, act="relu")     # z alone
        _check(base, prod * (z > 0), e, od)
    else:
        a, b = _mat(gen, rows, r, dt, scale=s), _mat(gen, cols, r, dt)
        prod, mag = a.double() @ b.double().t(), a.double().abs() @ b.double().abs().t()
        db, db2 = torch.zeros(rows, device="cuda"), torch.ones(rows, device="cuda")
        o2.copy_(base)
        C.dense_bwd_w(a, b, o1, ws, db=db)
        C.dense_bwd_w(a, b, o2, ws, db=db2, accumulate=True)
        e = _sum_tol(r, mag, od)
        want = prod + there
        _check(o2, want, e + 2.0 ** -23 * (want.abs() + there.abs()), od)
        sb, t = a.double().abs().sum(1), (r / 32 + 17) * 2.0 ** -23
        _check(db, a.double().sum(1), t * sb, torch.float32)
        _check(db2, a.double().sum(1) + 1, t * (sb + 1), torch.float32)
    _check(o1, prod, e, od)
    assert ws.status()[0] == 0
