"""Embedding lookup and its gradient against their definitions in float64.

Bounds, with u = 2^-24: the lookup rounds once in float32 (times scale) and once to its type. The gradient's sum over the
m tokens of a row has at most m + 8 float32 roundings, then those of the scale and of the addition to what is there.
Rounding to a type costs half a step, eps / 2.
"""

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
U = 2.0 ** -24


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
    """rows x cols values: tight rows, columns of a wider aligned buffer, or off the 16-byte grid; NaN around them."""
    v = (torch.randn(rows, cols, generator=gen, device="cuda") * scale).to(dt)
    if layout == "tight":
        return v
    wide = (cols + 63) // 64 * 64 + 64 if layout == "wide" else cols + 5
    buf = torch.full((rows, wide), float("nan"), dtype=dt, device="cuda")
    view = buf[:, 0:cols] if layout == "wide" else buf[:, 3:3 + cols]
    view.copy_(v)
    return view


def _untouched(t):
    buf = t._base
    if buf is None:
        return True
    mask = torch.ones_like(buf, dtype=torch.bool)
    o = t.storage_offset() % buf.stride(0)
    mask[:, o:o + t.shape[1]] = False
    return bool(buf[mask].isnan().all())


def _check(got, want, tol):
    dt = got.dtype
    tol = tol + torch.finfo(dt).eps / 2 * (want.abs() + tol) + (2.0 ** -25 if dt == torch.float16 else 0) + 1e-30
    bad = ~((got.double() - want).abs() <= tol)
    assert not bad.any(), (int(bad.sum()), float(((got.double() - want).abs() / tol).nan_to_num(1e30).max()))


def _tokens(gen, vocab, n, kind):
    if kind == "one":      # all the same
        t = torch.full((n,), vocab // 2, device="cuda")
    elif kind == "pad":    # a padded batch
        t = torch.randint(0, vocab, (n,), generator=gen, device="cuda")
        t[torch.rand(n, generator=gen, device="cuda") < 0.4] = -1
    elif kind == "skew":   # few of them come often
        t = (torch.rand(n, generator=gen, device="cuda") ** 6 * vocab).long().clamp_max(vocab - 1)
    elif kind == "distinct":
        t = torch.randperm(max(vocab, n), generator=gen, device="cuda")[:n] % vocab
    else:
        t = torch.randint(0, vocab, (n,), generator=gen, device="cuda")
    return t.to(torch.int32)


SHAPES = [(1, 1, 1), (5, 3, 7), (100, 64, 1), (100, 64, 64), (300, 130, 65), (1000, 1000, 777), (10000, 4096, 24),
          (32768, 520, 2048), (65536, 64, 5000), (70000, 33, 513), (257, 2049, 100), (64, 96, 9000), (3, 40, 20000)]


@pytest.mark.parametrize("vocab,d,n", SHAPES)
@pytest.mark.parametrize("table,dtype,layout", [("f32", "bf16", "tight"), ("bf16", "bf16", "odd"), ("f32", "f16", "wide"),
                                                ("f16", "f16", "tight"), ("bf16", "f32", "wide"), ("f32", "f32", "odd")])
def test_forward(C, vocab, d, n, table, dtype, layout):
    gen = _gen(vocab + d * 3 + n)
    w = _mat(gen, vocab, d, DT[table], layout)
    ws = C.EmbedWorkspace(vocab, d, n)
    for kind in ("any", "pad", "one"):
        tok = _tokens(gen, vocab, n, kind)
        x = _mat(gen, d, n, DT[dtype], layout)
        x.fill_(float("nan"))
        scale = 1.0 if kind == "pad" else d ** 0.5
        C.embed_fwd(w, tok, x, ws, scale=scale)
        s = float(torch.tensor(scale, dtype=torch.float32))
        want = torch.where(tok[:, None] >= 0, s * w[tok.long().clamp_min(0)].double(), 0.0).t()
        _check(x, want, U * want.abs())
        assert _untouched(x)
    assert ws.status()[0] == 0


@pytest.mark.parametrize("vocab,d,n", SHAPES)
@pytest.mark.parametrize("table,dtype,layout", [("f32", "bf16", "tight"), ("bf16", "bf16", "odd"), ("f32", "f16", "wide"),
                                                ("f16", "f16", "tight"), ("bf16", "f32", "wide"), ("f32", "f32", "odd")])
def test_backward(C, vocab, d, n, table, dtype, layout):
    gen = _gen(vocab + d * 3 + n)
    ws = C.EmbedWorkspace(vocab, d, n)
    for kind in ("any", "pad", "one", "skew", "distinct"):
        tok = _tokens(gen, vocab, n, kind)
        dx = _mat(gen, d, n, DT[dtype], layout)
        ok = tok >= 0
        index = tok.long().clamp_min(0)
        count = torch.zeros(vocab, dtype=torch.float64, device="cuda").index_add_(0, index, ok.double())
        s = float(torch.tensor(d ** 0.5, dtype=torch.float32))
        part = torch.where(ok[:, None], dx.double().t(), 0.0)
        total = torch.zeros(vocab, d, dtype=torch.float64, device="cuda").index_add_(0, index, part)
        size = torch.zeros(vocab, d, dtype=torch.float64, device="cuda").index_add_(0, index, part.abs())
        for accumulate in (False, True):
            dw = _mat(gen, vocab, d, DT[table], layout)
            before = dw.clone()
            if not accumulate:
                dw.fill_(float("nan"))
            C.embed_bwd(dx, tok, dw, ws, scale=d ** 0.5, accumulate=accumulate)
            want = s * total + (before.double() if accumulate else 0.0)
            tol = s * (count[:, None] + 9) * U * size + (U * want.abs() if accumulate else 0.0)
            if accumulate:
                assert torch.equal(dw[count == 0], before[count == 0])
            else:
                assert (dw[count == 0] == 0).all()
            _check(dw, want, tol)
            assert _untouched(dw)
            again = before.clone()
            C.embed_bwd(dx, tok, again, ws, scale=d ** 0.5, accumulate=accumulate)
            assert torch.equal(again, dw)   # repeats bit for bit, whatever the rows' stride
    assert ws.status()[0] == 0


def test_tokens_beyond_the_table(C):
    """They count as padding and are reported; every other token is as if they were not there."""
    gen = _gen(1)
    vocab, d, n = 50, 72, 130
    w, dx = _mat(gen, vocab, d, torch.float32), _mat(gen, d, n, torch.bfloat16)
    tok = _tokens(gen, vocab, n, "any")
    good = tok.clone()
    for at, bad in ((0, vocab), (17, 2 ** 31 - 1), (129, vocab + 5), (64, -2 ** 31)):
        tok[at] = bad
        good[at] = -1
    x, y = torch.empty(d, n, device="cuda"), torch.empty(d, n, device="cuda")
    a, b = torch.empty_like(w), torch.empty_like(w)
    ws = C.EmbedWorkspace(vocab, d, n)
    C.embed_fwd(w, good, y, ws)
    C.embed_bwd(dx, good, b, ws)
    assert ws.status()[0] == 0
    C.embed_fwd(w, tok, x, ws)
    assert ws.status()[0] == C.CSRT_DEV_INVALID
    ws.clear_status()
    C.embed_bwd(dx, tok, a, ws)
    assert ws.status()[0] == C.CSRT_DEV_INVALID
    assert torch.equal(x, y) and torch.equal(a, b)


def test_no_tokens(C):
    ws = C.EmbedWorkspace(20, 8, 0)
    none = torch.empty(0, dtype=torch.int32, device="cuda")
    C.embed_fwd(torch.zeros(20, 8, device="cuda"), none, torch.empty(8, 0, device="cuda"), ws)
    dw = torch.full((20, 8), 2.0, device="cuda")
    C.embed_bwd(torch.empty(8, 0, device="cuda"), none, dw, ws, accumulate=True)
    assert (dw == 2).all()
    C.embed_bwd(torch.empty(8, 0, device="cuda"), none, dw, ws)
    assert (dw == 0).all()


def test_rows_past_32_bits(C):
    """A table of more than 2^31 elements, and activations whose rows lie as far apart."""
    vocab, d, n = 70000, 40000, 20
    w = torch.zeros(vocab, d, dtype=torch.bfloat16, device="cuda")
    gen = _gen(2)
    tok = torch.tensor([69999, 5, 69999, 60000, 53688], dtype=torch.int32, device="cuda").repeat(4)
    w[69990:] = torch.randn(10, d, generator=gen, device="cuda").to(torch.bfloat16)
    x = torch.zeros(d * 60000, dtype=torch.bfloat16, device="cuda").view(d, 60000)[:, 100:100 + n]
    ws = C.EmbedWorkspace(vocab, d, n)
    C.embed_fwd(w, tok, x, ws)
    assert torch.equal(x, w[tok.long()].t())
    C.embed_bwd(x, tok, w, ws, scale=0.25)
    want = x[:, 0].double() * 2
    assert torch.equal(w[69999].double(), want)    # eight times a quarter, exact
    assert torch.equal(w[5], torch.zeros_like(w[5])) and (w[:69999].abs().amax() == 0)


def test_captured_on_another_stream(C):
    gen = _gen(4)
    vocab, d, n = 500, 136, 300
    w, dx = _mat(gen, vocab, d, torch.float32), _mat(gen, d, n, torch.bfloat16)
    tok = _tokens(gen, vocab, n, "skew")
    x, dw = torch.empty(d, n, dtype=torch.bfloat16, device="cuda"), torch.empty_like(w)
    ws = C.EmbedWorkspace(vocab, d, n)

    def run():
        C.embed_fwd(w, tok, x, ws, scale=2.0)
        C.embed_bwd(dx, tok, dw, ws, scale=2.0)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            run()
        for _ in range(2):
            tok.copy_(_tokens(gen, vocab, n, "any"))
            run()
            a, b = x.clone(), dw.clone()
            x.zero_(), dw.zero_()
            graph.replay()
            assert torch.equal(a, x) and torch.equal(b, dw)
    torch.cuda.current_stream().wait_stream(side)


# More tokens than are sorted by counting: one, two, three and four digits of the radix sort, and the last warp's share short
@pytest.mark.parametrize("vocab,d,n", [(255, 24, 16385), (300, 40, 20001), (70000, 16, 16385), (2 ** 24 + 5, 3, 16400)])
@pytest.mark.parametrize("table,dtype,layout", [("f32", "bf16", "tight"), ("bf16", "f32", "odd")])
def test_backward_sorted_by_digits(C, vocab, d, n, table, dtype, layout):
    test_backward(C, vocab, d, n, table, dtype, layout)


@pytest.mark.parametrize("vocab,n", [(50, 130), (50, 777), (300, 16385), (70000, 20000)])
@pytest.mark.parametrize("accumulate", [False, True])
def test_tokens_beyond_the_table_in_every_sort(C, vocab, n, accumulate):
    """Sorted in one launch, by counting and by digits: a token of vocab or more is padding, and reported."""
    gen = _gen(n)
    d = 24
    dx = _mat(gen, d, n, torch.bfloat16)
    tok = _tokens(gen, vocab, n, "pad")
    good = tok.clone()
    for at, bad in ((0, vocab), (n // 3, 2 ** 31 - 1), (n - 1, vocab + 5), (n // 2, -2 ** 31)):
        tok[at] = bad
        good[at] = -1
    a = _mat(gen, vocab, d, torch.float32)
    b = a.clone()
    ws = C.EmbedWorkspace(vocab, d, n)
    C.embed_bwd(dx, good, b, ws, accumulate=accumulate)
    assert ws.status()[0] == 0
    C.embed_bwd(dx, tok, a, ws, accumulate=accumulate)
    assert ws.status()[0] == C.CSRT_DEV_INVALID
    assert torch.equal(a, b)


def test_lookup_needs_no_workspace_for_its_tokens(C):
    """A program that only looks tokens up keeps the status words alone; the gradient asks for more."""
    gen = _gen(6)
    vocab, d, n = 90, 40, 3000
    w, tok = _mat(gen, vocab, d, torch.float32), _tokens(gen, vocab, n, "pad")
    ws = C.EmbedWorkspace(vocab, d, 0)
    assert ws.nbytes < 1 << 17
    x = torch.full((d, n), float("nan"), device="cuda")
    C.embed_fwd(w, tok, x, ws)
    assert torch.equal(x, torch.where(tok[:, None] >= 0, w[tok.long().clamp_min(0)], 0.0).t())
    tok[7] = vocab
    C.embed_fwd(w, tok, x, ws)
    assert ws.status()[0] == C.CSRT_DEV_INVALID
    with pytest.raises(C.CsrtError, match="workspace"):
        C.embed_bwd(x, tok, w, ws)
