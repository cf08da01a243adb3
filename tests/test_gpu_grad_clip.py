"""The global gradient norm and clipping against their definitions in float64.

Bounds: squares are summed in float32 over at most 128 terms (relative 2^-24 a term, all of one sign), then in float64,
and the norm is the root, rounded once: relative 65 x 2^-24 (a root halves the sum's error). The factor carries that and a
rounding, a product one more; the output rounds once to its type (half a step, eps / 2).
"""

import math

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


def _tensors(gen, shapes, dt, scale=1.0, odd=False):
    out = []
    for k, shape in enumerate(shapes):
        t = (torch.randn(shape, generator=gen, device="cuda") * scale).to(dt)
        if odd and k % 3 == 1:        # off the 16-byte grid
            flat = torch.empty(t.numel() + 1, dtype=dt, device="cuda")[1:].view(shape)
            t = flat.copy_(t)
        elif odd and k % 3 == 2 and len(shape) == 2:   # columns of a wider buffer
            wide = torch.full((shape[0], shape[1] + 9), float("nan"), dtype=dt, device="cuda")
            t = wide[:, 4:4 + shape[1]].copy_(t)
        out.append(t)
    return out


def _norm(ts):
    return math.sqrt(sum(float(t.double().square().sum()) for t in ts))


SETS = [[(1,)], [(1, 1), (0, 5), (7,)], [(784, 1024), (1024,), (1024, 784), (784,), (784,), (784,)] * 3,
        [(k + 1,) for k in range(40)], [(16384,), (16385,), (3, 16384), (33, 1000)],
        [(5000, 1), (1, 5000), (17, 31, 13), (), (70000, 3)], [(2000, 3001), (1000, 4096)], [(3, 7)] * 300, [(129, 513)] * 600]


@pytest.mark.parametrize("shapes", SETS, ids=[str(i) for i in range(len(SETS))])
@pytest.mark.parametrize("dt,out,odd", [("f32", "f32", False), ("f32", "bf16", True), ("bf16", "f32", False), ("f16", "f16", True),
                                        ("bf16", "bf16", False), ("f32", "f32", True)])
def test_norm_and_clip(C, shapes, dt, out, odd):
    gen = _gen(len(shapes))
    g = _tensors(gen, shapes, DT[dt], 0.1, odd)
    into = _tensors(gen, shapes, DT[out], 1.0, odd)
    want = _norm(g)
    ws, norm = C.GradWorkspace(), torch.zeros(2, device="cuda")
    C.grad_norm(g, norm, ws)
    assert abs(float(norm[0]) - want) <= 66 * U * want and float(norm[1]) == 1.0
    value = norm[0].clone()
    lists = C.TensorList(g), C.TensorList(into)
    for max_norm in (0.25 * want, 0.999 * want, 1.5 * want):
        norm.fill_(float("nan"))
        C.grad_clip(lists[0], max_norm, norm, ws, out=lists[1])
        assert norm[0] == value     # bit for bit
        factor = min(1.0, max_norm / want)
        assert abs(float(norm[1]) - factor) <= 68 * U * factor
        for a, b in zip(g, into):
            exact = a.double() * factor
            tol = (70 * U if factor < 1 else 0) * exact.abs()
            tol = tol + torch.finfo(b.dtype).eps / 2 * (exact.abs() + tol) + (2.0 ** -25 if b.dtype == torch.float16 else 0)
            assert ((b.double() - exact).abs() <= tol).all()
            if b._base is not None and b.dim() == 2 and b._base.dim() == 2:
                assert b._base[:, :4].isnan().all() and b._base[:, 4 + b.shape[1]:].isnan().all()
    # in place: the same values, and left alone where the norm is small enough
    separate = [t.clone() for t in g]
    C.grad_clip(g, 2 * want, norm, ws)
    assert all(torch.equal(a, b) for a, b in zip(g, separate))
    same_type = [torch.empty(t.shape, dtype=t.dtype, device="cuda") for t in g]
    C.grad_clip(g, 0.5 * want, norm, ws, out=same_type)
    C.grad_clip(g, 0.5 * want, norm, ws)
    assert all(torch.equal(a, b) for a, b in zip(g, same_type))
    assert ws.status()[0] == 0


@pytest.mark.parametrize("size", [1e-45, 1e-30, 1e-22, 1e-19, 1e15, 1e19, 3e38])
def test_values_whose_squares_leave_float32(C, size):
    """Tensors of tiny, ordinary and huge entries together: the norm is found wherever float32 holds it."""
    gen = _gen(3)
    base = torch.rand(3000, generator=gen, device="cuda") * 0.01
    t = torch.full((3000,), size, device="cuda") if size < 1e-40 else base * size
    g = [t, torch.zeros(70000, device="cuda"), t[:5].clone()]
    want = _norm(g)
    ws, norm = C.GradWorkspace(), torch.zeros(2, device="cuda")
    C.grad_norm(g, norm, ws)
    assert abs(float(norm[0]) - want) <= 66 * U * want + 2.0 ** -149
    if 1e-30 < want < 1e37:
        C.grad_clip(g, 0.5 * want, norm, ws)
        assert abs(_norm(g) - 0.5 * want) <= 140 * U * want + 1e-43 * 3000
    assert ws.status()[0] == 0


@pytest.mark.parametrize("bad", [float("inf"), float("-inf"), float("nan")])
def test_values_that_are_not_finite(C, bad):
    g = [torch.ones(1000, device="cuda"), torch.ones(64, 64, dtype=torch.bfloat16, device="cuda")]
    g[1][17, 5] = bad
    before = [t.clone() for t in g]
    ws, norm = C.GradWorkspace(), torch.zeros(2, device="cuda")
    C.grad_clip(g, 1.0, norm, ws)
    assert not math.isfinite(float(norm[0])) and float(norm[1]) == 1.0
    assert all(torch.equal(a.nan_to_num(7.0), b.nan_to_num(7.0)) for a, b in zip(g, before))
    assert ws.status()[0] == C.CSRT_DEV_NONFINITE
    ws.clear_status()
    g[1][17, 5] = 1
    C.grad_clip(g, 1.0, norm, ws)
    assert abs(_norm(g) - 1.0) < 0.01 and ws.status()[0] == 0


def test_nothing(C):
    ws, norm = C.GradWorkspace(), torch.full((2,), 5.0, device="cuda")
    C.grad_clip([], 1.0, norm, ws)
    assert norm.tolist() == [0.0, 1.0]
    C.grad_clip([torch.empty(0, 7, device="cuda"), torch.zeros(9, device="cuda")], 1.0, norm, ws)
    assert norm.tolist() == [0.0, 1.0] and ws.status()[0] == 0


def test_more_than_2_31_elements(C):
    """One tensor past 32-bit counts, its entries beyond them the only ones that are not zero."""
    t = torch.zeros(3, 715850000, dtype=torch.bfloat16, device="cuda")
    assert t.numel() > 2 ** 31 + 2 ** 16
    t.view(-1)[-5:] = 3.0
    ws, norm = C.GradWorkspace(), torch.zeros(2, device="cuda")
    C.grad_clip([t], 1.0, norm, ws)
    assert abs(float(norm[0]) - math.sqrt(45)) < 1e-5
    got = t.view(-1)[-5:].double()
    assert ((got - 3 / math.sqrt(45)).abs() <= 2.0 ** -8 * 0.45 + 1e-6).all()


def test_captured_on_another_stream(C):
    gen = _gen(8)
    g = _tensors(gen, [(300, 700), (700,), (64, 33)], torch.float32)
    into = [torch.empty_like(t) for t in g]
    ws, norm = C.GradWorkspace(), torch.zeros(2, device="cuda")
    gl, ol = C.TensorList(g), C.TensorList(into)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        C.grad_clip(gl, 2.0, norm, ws, out=ol)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            C.grad_clip(gl, 2.0, norm, ws, out=ol)
        for k in (1.0, 1e-3, 5.0):
            for t in g:
                t.normal_(generator=gen).mul_(k)
            C.grad_clip(gl, 2.0, norm, ws, out=ol)
            want = [t.clone() for t in into] + [norm.clone()]
            for t in into + [norm]:
                t.zero_()
            graph.replay()
            assert all(torch.equal(a, b) for a, b in zip(want, into + [norm]))
    torch.cuda.current_stream().wait_stream(side)
    assert ws.status()[0] == 0


def test_one_memory_twice_is_not_written(C):
    """A tensor that is listed twice counts twice in a norm, and is refused where it would be scaled twice."""
    t = torch.full((40, 30), 2.0, device="cuda")
    ws, norm = C.GradWorkspace(), torch.zeros(2, device="cuda")
    C.grad_norm([t, t], norm, ws)
    assert abs(float(norm[0]) - math.sqrt(2 * 1200 * 4)) < 1e-3
    for pair in ([t, t], [t, t[3:7]], [t.view(-1)[:100], t.view(-1)[99:200]]):
        with pytest.raises(ValueError, match="overlap"):
            C.grad_clip(pair, 1.0, norm, ws)
    assert (t == 2).all()
    out = [torch.empty_like(t), torch.empty_like(t)]
    C.grad_clip([t, t], 1.0, norm, ws, out=out)
    assert torch.equal(out[0], out[1]) and float(out[0][0, 0]) < 1
    C.grad_clip([t.view(-1)[:100], t.view(-1)[100:200]], 1.0, norm, ws)   # side by side


def test_first_call_is_captured(C):
    """Nothing has to run eagerly first (in a process of its own)."""
    import subprocess
    import sys
    code = """
import torch
from paper_1905_07931_gb300 import csrtrain as C
g = [torch.ones(300, 300, device="cuda"), torch.ones(70000, 200, device="cuda")]
ws, norm = C.GradWorkspace(), torch.zeros(2, device="cuda")
y = torch.randn(520, 96, device="cuda").bfloat16(); h, v = torch.empty_like(y), torch.empty_like(y)
rstd = torch.empty(96, device="cuda")
wsn = C.BlockNormWorkspace(520, 96)
dr, dw = torch.empty_like(y), torch.empty(520, device="cuda")
N = C.Norm("rms", rstd=rstd, dweight=dw)
table, tok = torch.randn(50, 520, device="cuda"), torch.randint(0, 50, (96,), device="cuda").int()
wse = C.EmbedWorkspace(50, 520, 96)
torch.cuda.synchronize()
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    C.embed_fwd(table, tok, y, wse)
    C.block_norm_fwd(y, None, h, v, pre=N)
    C.block_norm_bwd(v, None, h, None, dr, None, wsn, pre=N)
    C.embed_bwd(dr, tok, table, wse, accumulate=True)
    C.grad_clip(g[:1], 1.0, norm, ws)
    C.grad_clip(g, 1.0, norm, ws)
graph.replay()
torch.cuda.synchronize()
assert all(w.status()[0] == 0 for w in (ws, wsn, wse))
assert abs(float((g[0].double() ** 2).sum() + (g[1].double() ** 2).sum()) - 1) < 1e-3
print("captured")
"""
    r = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, timeout=110)
    assert r.returncode == 0 and "captured" in r.stdout, r.stderr


def test_wait_that_runs_out(C):
    """A count of arrived sums that cannot become complete (the test begins it far too high): the call of one launch gives
    up and says so, out stays as it was, and the workspace serves the next calls, in one launch and in two."""
    gen = _gen(12)
    small, large = _tensors(gen, [(300, 100), (7,)], torch.float32), _tensors(gen, [(3000, 1000), (5,)], torch.float32)
    ws, norm = C.GradWorkspace(), torch.zeros(2, device="cuda")
    counters = ws.buf[256:264].view(torch.int32)   # behind the status words
    C.grad_clip(small, 1e6, norm, ws)
    assert counters.tolist() == [0, 0]
    counters[0] = 1000
    before = [t.clone() for t in small]
    C.grad_clip(small, 1.0, norm, ws)
    assert ws.status()[0] == C.CSRT_DEV_TIMEOUT
    assert norm.isnan().all() and all(torch.equal(a, b) for a, b in zip(small, before))
    assert counters.tolist() == [0, 0]
    ws.clear_status()
    for g in (large, small, large):
        want = _norm(g)
        C.grad_clip(g, 0.5 * want, norm, ws)
        assert abs(float(norm[0]) - want) <= 66 * U * want and abs(_norm(g) - 0.5 * want) <= 140 * U * want
    assert ws.status()[0] == 0


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("numel,offset,steps", [(3 * 8192 * 304, 0, 6.5), (8192 * 4096 + 3, 0, 6.5), (8192 * 512 + 1000, 1, 17)])
def test_norms_of_long_sums(C, dt, numel, offset, steps):
    """The squares of 32 entries are summed in float32, all else in float64. Whole vectors: eight products on each of four sums
    (a rounding each), two additions, one more for an entry behind the last vector: 11 x 2^-24 of the sum, half of it of the
    root, which is rounded once. Off the 16-byte grid: 32 roundings one after the other, and the root's."""
    gen = _gen(numel % 1000)
    t = torch.rand(numel + offset, generator=gen, device="cuda").to(DT[dt])[offset:]
    want = float(t.double().square().sum()) ** 0.5
    ws, norm = C.GradWorkspace(), torch.zeros(2, device="cuda")
    C.grad_norm([t], norm, ws)
    assert abs(float(norm[0]) - want) <= steps * U * 1.0001 * want
    C.grad_clip([t], 0.5 * want, norm, ws, out=[torch.empty(numel, device="cuda")])
    assert abs(float(norm[0]) - want) <= steps * U * 1.0001 * want


def test_norm_beyond_float32(C):
    """Finite entries whose norm float32 does not hold: it is returned as infinite, and they are clipped as any others."""
    g = [torch.full((1000,), 3e38, device="cuda"), torch.full((40, 50), -2e38, device="cuda")]
    want = _norm(g)
    ws, norm = C.GradWorkspace(), torch.zeros(2, device="cuda")
    out = [torch.empty_like(t) for t in g]
    C.grad_clip(g, 1e38, norm, ws, out=out)
    assert float(norm[0]) == math.inf and abs(float(norm[1]) - 1e38 / want) <= 66 * U * 1e38 / want
    for a, b in zip(g, out):
        exact = a.double() * 1e38 / want
        assert ((b.double() - exact).abs() <= 70 * U * exact.abs()).all()
    assert ws.status()[0] == 0
