"""The orthogonalised update against its iteration in float64.

Bounds. The products' operands are float16 (2^-12 of an entry on average 1.4e-4 to 2e-4 of a matrix in the 2-norm):
three of them a step, five steps, and the polynomial's slope is at most 1.6 where singular values have arrived: about
sqrt(15) x 2e-4 x 1.6 = 1.3e-3 of o in the 2-norm where roundings add at random; 2e-3 is allowed. bfloat16 results add
their own rounding, 1.7e-3 in the 2-norm (uniform within 2^-9): 3e-3 in all. The momentum is exact float32 arithmetic.
"""

import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

A, B, CC = 3.4445, -4.7750, 2.0315


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


def _exact(u, steps, eps, scale):
    out = torch.empty_like(u)
    for i in range(u.shape[0]):
        x = u[i] / max(float(u[i].norm()), eps)
        tall = x.shape[0] > x.shape[1]
        x = x.t() if tall else x
        for _ in range(steps):
            a = x @ x.t()
            x = A * x + (B * a + CC * (a @ a)) @ x
        out[i] = scale * (x.t() if tall else x)
    return out


def _rel(got, want):
    return float((got.double() - want).norm() / want.norm())


SHAPES = [(1, 1, 1), (1, 1, 7), (2, 5, 1), (3, 3, 9), (1, 64, 64), (5, 64, 65), (1, 65, 130), (4, 129, 33), (1, 300, 784),
          (1, 784, 300), (2, 200, 1000), (12, 96, 160), (1, 128, 4100), (1, 1000, 1024), (3, 700, 515), (2, 1300, 2051),
          (1, 2050, 3000), (6, 256, 2048), (3, 2048, 1024)]


@pytest.mark.parametrize("batch,m,k", SHAPES)
@pytest.mark.parametrize("gdt,odt,nesterov", [(torch.float32, torch.float32, True), (torch.bfloat16, torch.bfloat16, True),
                                              (torch.float32, torch.bfloat16, False)])
def test_direction_and_momentum(C, batch, m, k, gdt, odt, nesterov):
    gen = _gen(batch * 10007 + m * 31 + k)
    g = (torch.randn(batch, m, k, generator=gen, device="cuda") * 1e-3).to(gdt)
    mom = torch.randn(batch, m, k, generator=gen, device="cuda") * 3e-3
    beta, scale = 0.95, 0.2 * math.sqrt(max(m, k))
    bt = torch.tensor(beta, dtype=torch.float32, device="cuda")
    want_mom = mom * bt + g.float()
    u = g.float() + bt * want_mom if nesterov else want_mom
    o = torch.empty(batch, m, k, dtype=odt, device="cuda")
    ws = C.OrthogonalizeWorkspace(batch, m, k)
    C.orthogonalize(g, o, ws, momentum=mom, beta=beta, nesterov=nesterov, scale=scale)
    assert torch.equal(mom, want_mom)
    assert _rel(o, _exact(u.double(), 5, 1e-7, scale)) <= (2e-3 if odt == torch.float32 else 3e-3)
    assert ws.status()[0] == 0


@pytest.mark.parametrize("steps", [0, 1, 2, 3, 8])
def test_steps(C, steps):
    g = torch.randn(2, 90, 150, generator=_gen(steps), device="cuda")
    o, ws = torch.empty_like(g), C.OrthogonalizeWorkspace(2, 90, 150)
    C.orthogonalize(g, o, ws, steps=steps, scale=2.0)
    assert _rel(o, _exact(g.double(), steps, 1e-7, 2.0)) <= (1e-6 if steps == 0 else 2e-3)


def test_singular_values_arrive_near_one(C):
    g = torch.randn(400, 900, generator=_gen(1), device="cuda")
    o, ws = torch.empty_like(g), C.OrthogonalizeWorkspace(1, 400, 900)
    C.orthogonalize(g, o, ws)
    s = torch.linalg.svdvals(o.double())
    assert 0.6 < float(s.min()) and float(s.max()) < 1.3


@pytest.mark.parametrize("where", ["g", "o", "both"])
@pytest.mark.parametrize("m,k", [(37, 53), (130, 258)])
def test_strided_and_unaligned(C, where, m, k):
    gen, batch = _gen(2), 3
    v = torch.randn(batch, m, k, generator=gen, device="cuda")
    g, o = v, torch.empty(batch, m, k, device="cuda")
    if where in ("g", "both"):
        g = torch.full((batch, m + 2, k + 7), float("nan"), device="cuda")[:, 1:m + 1, 3:3 + k]
        g.copy_(v)
    if where in ("o", "both"):   # matrices side by side in one wide buffer: rows interleave
        o = torch.zeros(m, batch, k + 1, device="cuda").permute(1, 0, 2)[:, :, :k]
    ws = C.OrthogonalizeWorkspace(batch, m, k)
    C.orthogonalize(g, o, ws)
    assert _rel(o, _exact(v.double(), 5, 1e-7, 1.0)) <= 2e-3


@pytest.mark.parametrize("scale", [1e-30, 1e-12, 1e12, 1e30])
def test_norms_far_from_one(C, scale):
    v = torch.randn(1, 100, 140, generator=_gen(6), device="cuda")
    o, ws = torch.empty_like(v), C.OrthogonalizeWorkspace(1, 100, 140)
    C.orthogonalize((v.double() * scale).float(), o, ws, eps=1e-38)
    assert _rel(o, _exact(v.double(), 5, 1e-38, 1.0)) <= 2e-3


def test_zero_and_not_a_number(C):
    g = torch.randn(4, 80, 96, generator=_gen(7), device="cuda")
    g[1] = 0
    g[2, 5, 6] = float("nan")
    g[3, 7, 8] = float("inf")
    o, ws = torch.empty_like(g), C.OrthogonalizeWorkspace(4, 80, 96)
    C.orthogonalize(g, o, ws)
    assert bool((o[1] == 0).all()) and bool(o[2].isnan().all()) and bool(o[3].isnan().all())
    assert _rel(o[:1], _exact(g[:1].double(), 5, 1e-7, 1.0)) <= 2e-3   # the others are not touched by them


@pytest.mark.parametrize("spread", [30.0, 300.0])
def test_strong_directions(C, spread):
    """A few directions far above the rest, as gradients have them: the rest still comes out."""
    gen = _gen(11)
    u, _ = torch.linalg.qr(torch.randn(256, 256, generator=gen, device="cuda").double())
    v, _ = torch.linalg.qr(torch.randn(512, 256, generator=gen, device="cuda").double())
    s = torch.ones(256, device="cuda").double()
    s[:6] = spread
    g = ((u * s) @ v.t()).float()[None].contiguous()
    o, ws = torch.empty_like(g), C.OrthogonalizeWorkspace(1, 256, 512)
    C.orthogonalize(g, o, ws, steps=7)
    assert _rel(o, _exact(g.double(), 7, 1e-7, 1.0)) <= 5e-3


@pytest.mark.parametrize("rank,m,k", [(1, 60, 90), (16, 128, 200), (64, 300, 500), (200, 512, 1024)])
def test_rank_deficient(C, rank, m, k):
    """A gradient of few samples has singular values at zero, where the iteration multiplies whatever a step's rounding
    leaves by a = 3.4445 in each later step: 2e-4 x |b| of at most 1 in the 2-norm, times 3.4445^(4 - step), sums to
    0.19 against sqrt(rank) of the result, for each of the three operands at random: 0.33 / sqrt(rank)."""
    gen = _gen(rank)
    g = (torch.randn(m, rank, generator=gen, device="cuda") @ torch.randn(rank, k, generator=gen, device="cuda"))[None]
    o, ws = torch.empty_like(g), C.OrthogonalizeWorkspace(1, m, k)
    C.orthogonalize(g, o, ws)
    assert _rel(o, _exact(g.double(), 5, 1e-7, 1.0)) <= 0.33 / math.sqrt(rank)


def test_repeats_bit_for_bit_and_in_a_graph(C):
    g = torch.randn(3, 300, 520, generator=_gen(13), device="cuda").bfloat16()
    ws, outs = C.OrthogonalizeWorkspace(3, 300, 520), []
    for _ in range(4):
        o = torch.empty_like(g)
        C.orthogonalize(g, o, ws)
        outs.append(o)
    assert all(torch.equal(o, outs[0]) for o in outs)
    o, graph = torch.zeros_like(g), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        C.orthogonalize(g, o, ws)
    for _ in range(2):
        o.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(o, outs[0])


def test_two_streams_at_once(C):
    """Two calls on two streams (a workspace each): the cooperative launches neither mix nor wait for one another's units."""
    gs = [torch.randn(2, 260, 700, generator=_gen(20 + i), device="cuda") for i in range(2)]
    wss = [C.OrthogonalizeWorkspace(2, 260, 700) for _ in range(2)]
    outs = [torch.empty_like(g) for g in gs]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(5):
        for g, o, ws, s in zip(gs, outs, wss, streams):
            C.orthogonalize(g, o, ws, stream=s)
    torch.cuda.synchronize()
    for g, o, ws in zip(gs, outs, wss):
        assert _rel(o, _exact(g.double(), 5, 1e-7, 1.0)) <= 2e-3
        assert ws.status()[0] == 0


def test_binding_refuses(C):
    g = torch.zeros(4, 6, device="cuda")
    ws = C.OrthogonalizeWorkspace(1, 4, 6)
    with pytest.raises(ValueError, match="one shape"):
        C.orthogonalize(g, torch.zeros(6, 4, device="cuda"), ws)
    with pytest.raises(ValueError, match="momentum"):
        C.orthogonalize(g, torch.empty_like(g), ws, momentum=torch.zeros(4, 5, device="cuda"))
    with pytest.raises(C.CsrtError, match="workspace has"):
        C.orthogonalize(torch.zeros(300, 500, device="cuda"), torch.zeros(300, 500, device="cuda"),
                        C.DenseWorkspace(1, 1, 1))
    with pytest.raises(C.CsrtError, match="overlaps g"):
        C.orthogonalize(g, g, ws)


# --- with the compressed layers ---------------------------------------------

def test_sparse_net_trains_along_orthogonalised_directions(C):
    """SparseNet(optimizer="muon"): each layer's new CSR is the prox step of the direction that the call gave for the
    layer (the direction itself is checked above, also for gradients of low rank such as these)."""
    import numpy as np

    import oracle as O
    from paper_1905_07931_gb300 import synth
    from paper_1905_07931_gb300.train import SparseNet, mlp_layers
    cfg = synth.mlp(seed=3, batch=64, sizes=(96, 80, 10), densities=(0.3, 0.4))
    net = SparseNet(mlp_layers(2), cfg["W"], cfg["b"], 64, (96,), optimizer="muon", grad_per_layer=True)
    net.x_in.copy_(torch.from_numpy(cfg["X"]))
    net.labels.copy_(torch.from_numpy(cfg["labels"]))
    eta, lam = 0.02, 0.05
    losses = []
    for t in range(6):
        old = [net.weights(i).to_host()[0] for i in range(2)]
        losses.append(float(net.step("prox", eta, lam)[0].item()))
        assert net.status()[0] == 0
        for i, L in enumerate(net.params):
            w = O.CSR(L["W"][0].rows, L["W"][0].cols, *old[i])
            want = O.prox_update_compact(w, L["o"].cpu().numpy(), np.float32(eta), np.float32(lam))
            rp, ci, v = net.weights(i).to_host()[0]
            np.testing.assert_array_equal(rp, want.row_ptr)
            np.testing.assert_array_equal(ci, want.col_idx)
            np.testing.assert_array_equal(v.view(np.uint32), want.val.astype(np.float32).view(np.uint32))
    assert losses[-1] < losses[0]


def test_residual_net_gradients_and_training(C):
    """The example's gradients against float64 backpropagation (bfloat16 activations: some eight roundings of 2^-9 on
    the way, 2.5e-2 of a gradient's norm allowed), and that training brings the loss down."""
    from paper_1905_07931_gb300.residual import ResidualNet
    net = ResidualNet(72, 104, 2, 10, 88, seed=2)
    gen = _gen(40)
    centres = torch.randn(72, 10, generator=gen, device="cuda")
    y = torch.randint(0, 10, (88,), generator=gen, device="cuda")
    net.x[0].copy_(0.5 * centres[:, y] + torch.randn(72, 88, generator=gen, device="cuda"))
    net.labels.copy_(y)
    wc = torch.zeros(10, 72, dtype=torch.float64, device="cuda")
    (rp, ci, v), _ = net.wc[0].to_host()
    for r in range(10):
        for j in range(rp[r], rp[r + 1]):
            wc[r, ci[j]] = float(v[j])
    p = [net.w1h.double().requires_grad_(), net.w2h.double().requires_grad_(), net.b1.double().requires_grad_(),
         net.b2.double().requires_grad_(), wc.requires_grad_()]
    x = net.x[0].double()
    for i in range(2):
        z = p[0][i] @ x + p[2][i][:, None]
        x = x + p[1][i] @ torch.nn.functional.gelu(z, approximate="tanh") + p[3][i][:, None]
    loss = torch.nn.functional.cross_entropy((p[4] @ x).t(), y)
    loss.backward()
    first = float(net.step(0.0, 0.0)[0].item())
    assert abs(first - float(loss)) <= 2e-2 * float(loss)
    for got, want in zip((net.g1, net.g2, net.db1, net.db2, net.gc), p):
        assert _rel(got, want.grad) <= 2.5e-2
    for _ in range(20):
        last = float(net.step(0.02, 0.05)[0].item())
    assert last < 0.7 * first and net.status() == 0


@pytest.mark.parametrize("m,k", [(96, 160), (65, 33)])
@pytest.mark.parametrize("odt", [torch.float32, torch.bfloat16])
def test_matrices_far_apart(C, m, k, odt):
    """A batch whose second matrix lies past 2^31 elements gives the bits of the same matrices close together."""
    gen = _gen(m + k)
    far = 2 ** 31 + 64
    g = torch.randn(2, m, k, generator=gen, device="cuda")
    bg = torch.empty(far + m * k, device="cuda")
    bo = torch.empty(far + m * k, dtype=odt, device="cuda")
    gf, of = bg.as_strided((2, m, k), (far, k, 1)), bo.as_strided((2, m, k), (far, k, 1))
    gf.copy_(g)
    o = torch.empty(2, m, k, dtype=odt, device="cuda")
    ws = C.OrthogonalizeWorkspace(2, m, k)
    ma, mb = torch.zeros(2, m, k, device="cuda"), torch.zeros(2, m, k, device="cuda")
    C.orthogonalize(g, o, ws, momentum=ma)
    C.orthogonalize(gf, of, ws, momentum=mb)
    assert torch.equal(o, of) and torch.equal(ma, mb)


@pytest.mark.parametrize("batch,m,k", [(1, 3000, 4000), (1, 4001, 2900), (4, 1500, 2000)])
@pytest.mark.parametrize("odt", [torch.float32, torch.bfloat16])
def test_large_matrices(C, batch, m, k, odt):
    """Sizes from which on the largest tiles serve, their left-over tiles in slices where there is one matrix."""
    gen = _gen(batch + m + k)
    g = torch.randn(batch, m, k, generator=gen, device="cuda")
    o, o2 = torch.empty(batch, m, k, dtype=odt, device="cuda"), torch.empty(batch, m, k, dtype=odt, device="cuda")
    ws = C.OrthogonalizeWorkspace(batch, m, k)
    C.orthogonalize(g, o, ws, scale=0.5)
    C.orthogonalize(g, o2, ws, scale=0.5)
    assert torch.equal(o, o2)
    assert _rel(o, _exact(g.double(), 5, 1e-7, 0.5)) <= (2e-3 if odt == torch.float32 else 3e-3)


@pytest.mark.parametrize("m,k", [(40, 60), (33, 7)])
@pytest.mark.parametrize("steps", [0, 5])
def test_factors_out_of_float32_range(C, m, k, steps):
    """eps and norms so small (or, with no steps, a result so far from the norm) that the factor between u and o is no
    float32: a zero matrix stays zero, others come out as from the definition."""
    # entries that float32 holds exactly: 2^-120 times a float16
    v = torch.randn(1, m, k, generator=_gen(m + steps), device="cuda").half().double()
    cases = [(0.0, 1e-38, 1.0), (0.0, 1e-45, 8.0), (2.0 ** -120, 1e-38, 1.0), (2.0 ** -120, 1e-45, 8.0)]
    if steps == 0:
        cases += [(2.0 ** -120, 1e-45, 3e38), (2.0 ** 110, 1e-7, 2e-5), (2.0 ** 110, 1e-7, 1e-6)]
    ws = C.OrthogonalizeWorkspace(1, m, k)
    for factor, eps, scale in cases:
        g = (v * factor).float()
        assert torch.equal(g.double(), v * factor)
        o = torch.full_like(g, float("nan"))
        C.orthogonalize(g, o, ws, eps=eps, steps=steps, scale=scale)
        if factor == 0.0:
            assert bool((o == 0).all())
        else:   # without steps: the float32 factor's and the product's roundings, and float32's smallest step
            want = _exact(g.double(), steps, 0.0, scale)
            assert bool(o.isfinite().all())
            if steps == 0:
                assert bool(((o.double() - want).abs() <= 2.0 ** -22 * want.abs() + 2.0 ** -149).all())
            else:
                assert _rel(o, want) <= 2e-3


@pytest.mark.parametrize("batch,m,k", [(2, 64, 20000), (2, 130, 40000), (2, 64, 1200000), (2, 1200000, 40), (1, 33, 4000000),
                                       (3, 300, 300000)])
def test_very_long_matrices(C, batch, m, k):
    """The Gram matrix's sums of squares, all of one sign, over a long side: 1.2e-4 of A at most (the tensor core's own
    sums stop after 16384 terms), within what the bounds above allow."""
    g = torch.randn(batch, m, k, generator=_gen(batch + m + k), device="cuda")
    o, ws = torch.empty_like(g), C.OrthogonalizeWorkspace(batch, m, k)
    C.orthogonalize(g, o, ws)
    assert ws.status()[0] == 0
    for i in range(batch):
        assert _rel(o[i:i + 1], _exact(g[i:i + 1].double(), 5, 1e-7, 1.0)) <= 2e-3


def test_short_side_of_many_thousands(C):
    """All three products have long sums. u = Q1 diag(s) Q2^T, so that the iteration acts on s alone. Where u is zero the
    roundings grow as csrtrain.h says: a few 1e-3."""
    n, r = 16640, 512
    gen = _gen(77)
    q1, _ = torch.linalg.qr(torch.randn(n, r, generator=gen, device="cuda").double())
    q2, _ = torch.linalg.qr(torch.randn(n, r, generator=gen, device="cuda").double())
    s = 1.0 + torch.rand(r, generator=gen, device="cuda").double()
    g = ((q1 * s) @ q2.t()).float()[None].contiguous()
    o, ws = torch.empty_like(g), C.OrthogonalizeWorkspace(1, n, n)
    C.orthogonalize(g, o, ws)
    p = s / s.norm()
    for _ in range(5):
        p = A * p + B * p ** 3 + CC * p ** 5
    want = (q1 * p) @ q2.t()
    assert ws.status()[0] == 0
    assert _rel(o[0], want) <= 4e-3


def test_a_row_of_nearly_2_31_elements(C):
    """A vector has one singular value: o is the iteration's scalar times the unit vector."""
    n = 2 ** 31 - 1
    m, k = 1, n
    g = torch.zeros(m, k, device="cuda")
    o = torch.full((m, k), float("nan"), dtype=torch.bfloat16, device="cuda")
    at = torch.tensor([0, 5, 2 ** 30, n - 300, n - 9, n - 1], device="cuda")
    g.view(-1)[at] = torch.tensor([3.0, -1.0, 2.0, -4.0, 0.5, 1.5], device="cuda")
    ws = C.OrthogonalizeWorkspace(1, m, k)
    C.orthogonalize(g, o, ws, steps=2)
    v = g.view(-1)[at].double()
    p = 1.0
    for _ in range(2):
        p = A * p + B * p ** 3 + CC * p ** 5
    assert ws.status()[0] == 0
    # X's float16 copies, the Gram sum and o's own rounding
    assert _rel(o.view(-1)[at], p * v / v.norm()) <= 3e-3
    assert int(torch.count_nonzero(o)) == 6
    del g, o, ws
    torch.cuda.empty_cache()


def test_a_batch_of_the_longest_rows(C):
    """Two rows of nearly 2^31 elements in one call: their sums are shared among the SMs, so that no unit waits for seconds."""
    n, batch = 2 ** 31 - 1, 2
    g = torch.zeros(batch, 1, n, device="cuda")
    o = torch.full((batch, 1, n), float("nan"), dtype=torch.bfloat16, device="cuda")
    at = torch.tensor([0, 2 ** 30, n - 9, n - 1], device="cuda")
    vals = torch.tensor([[3.0, -1.0, 2.0, 0.5], [1.0, 4.0, -2.0, 8.0]], device="cuda")
    for i in range(batch):
        g[i, 0, at] = vals[i]
    ws = C.OrthogonalizeWorkspace(batch, 1, n)
    C.orthogonalize(g, o, ws, steps=1)
    assert ws.status()[0] == 0
    for i in range(batch):
        v = vals[i].double() / vals[i].double().norm()
        assert _rel(o[i, 0, at], (A + B + CC) * v) <= 3e-3
    assert int(torch.count_nonzero(o)) == 8
    del g, o, ws
    torch.cuda.empty_cache()


@pytest.mark.parametrize("odt", [torch.float32, torch.bfloat16])
def test_long_batches_one_by_one(C, odt):
    """Matrices that a call takes one after the other give what each gives by itself, bit for bit."""
    batch, k = 2, 2 ** 26 + 64
    g = torch.randn(batch, 2, k, generator=_gen(91), device="cuda")
    o, ws = torch.empty(batch, 2, k, dtype=odt, device="cuda"), C.OrthogonalizeWorkspace(batch, 2, k)
    C.orthogonalize(g, o, ws, steps=2)
    one, wso = torch.empty(2, k, dtype=odt, device="cuda"), C.OrthogonalizeWorkspace(1, 2, k)
    for i in range(batch):
        C.orthogonalize(g[i], one, wso, steps=2)
        assert torch.equal(one, o[i])
    assert ws.status()[0] == 0
    assert _rel(o, _exact(g.double(), 2, 1e-7, 1.0)) <= (2e-3 if odt == torch.float32 else 3e-3)
    del g, o, ws, one, wso
    torch.cuda.empty_cache()


@pytest.mark.parametrize("m,k", [(33, 5), (64, 65), (300, 130), (1000, 1001), (2000, 3003)])
@pytest.mark.parametrize("odt", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("batch", [1, 2])
def test_nothing_is_written_between_rows(C, m, k, odt, batch):
    """o as the first columns of aligned wider rows, with a row between the matrices: all else stays as it is."""
    g = torch.randn(batch, m, k, generator=_gen(m + k), device="cuda")
    buf = torch.full((batch, m + 1, (k + 63) // 64 * 64 + 64), 7.0, dtype=odt, device="cuda")
    o, ws = buf[:, :m, :k], C.OrthogonalizeWorkspace(batch, m, k)
    C.orthogonalize(g, o, ws)
    assert _rel(o, _exact(g.double(), 5, 1e-7, 1.0)) <= (2e-3 if odt == torch.float32 else 3e-3)
    assert bool((buf[:, m] == 7).all()) and bool((buf[:, :, k:] == 7).all())


@pytest.mark.parametrize("rank,m,k", [(1, 60, 90), (16, 128, 200), (64, 300, 500), (200, 512, 1024), (1, 10, 72), (4, 10, 72),
                                      (8, 784, 300), (32, 1500, 2000)])
def test_rank_deficient_within_what_the_header_says(C, rank, m, k):
    """In the row and column space of u the bound is the one for full rank. Outside, a step's rounding of A and B (1.4e-4
    of an entry, rms) times X has 2.4e-4 |A| sqrt(rank / s) |X| left, s the short side and A, X of norm 1 / sqrt(rank) and
    1 / sqrt(rank) a direction at the first step; times |b| for either, times 3.4445^4 and what later steps add (146), over
    the result's sqrt(rank): 0.14 / (rank sqrt(s)). Beside that the header's 3e-3, 4e-3 with a margin."""
    gen = _gen(rank + m)
    g = (torch.randn(m, rank, generator=gen, device="cuda") @ torch.randn(rank, k, generator=gen, device="cuda"))[None]
    o, ws = torch.empty_like(g), C.OrthogonalizeWorkspace(1, m, k)
    C.orthogonalize(g, o, ws)
    want = _exact(g.double(), 5, 1e-7, 1.0)
    assert _rel(o, want) <= 4e-3 + 0.14 / (rank * math.sqrt(min(m, k)))
    u, _, vt = torch.linalg.svd(g[0].double(), full_matrices=False)
    u, vt = u[:, :rank], vt[:rank]
    err = u @ (u.t() @ (o[0].double() - want[0]) @ vt.t()) @ vt
    assert float(err.norm() / want.norm()) <= 2e-3


@pytest.mark.parametrize("workload", ["mlp", "lenet"])
def test_sparse_net_updates_on_a_second_stream(C, workload):
    """SparseNet(optimizer="muon") with each layer's update beside the backward pass gives the bits of one stream, on fc
    and on conv layers."""
    import numpy as np

    from paper_1905_07931_gb300 import synth
    from paper_1905_07931_gb300.train import SparseNet, lenet_layers, mlp_layers
    if workload == "mlp":
        cfg = synth.mlp(seed=5, batch=64, sizes=(200, 120, 84, 10), densities=(0.3, 0.3, 0.5))
        layers, shape, count = mlp_layers(3), (200,), 3
    else:
        cfg = synth.lenet(seed=5, batch=16)
        layers, shape, count = lenet_layers(), (1, 28, 28), len(cfg["W"])
    batch = cfg["labels"].shape[0]
    nets = []
    for ov in (False, True):
        net = SparseNet(layers, cfg["W"], cfg["b"], batch, shape, optimizer="muon", overlap=ov)
        net.x_in.copy_(torch.from_numpy(np.ascontiguousarray(cfg["X"])).view_as(net.x_in))
        net.labels.copy_(torch.from_numpy(cfg["labels"]))
        nets.append(net)
    losses = []
    for _ in range(4):
        pair = [float(net.step("prox", 0.01, 0.05)[0].item()) for net in nets]
        torch.cuda.synchronize()
        assert pair[0] == pair[1] and math.isfinite(pair[0])
        losses.append(pair[0])
        assert all(net.status()[0] == 0 for net in nets)
        for i in range(count):
            for a, b in zip(nets[0].weights(i).to_host()[0], nets[1].weights(i).to_host()[0]):
                np.testing.assert_array_equal(a.view(np.uint32), b.view(np.uint32))
            assert torch.equal(nets[0].params[i]["m"], nets[1].params[i]["m"])
    assert losses[-1] < losses[0]
