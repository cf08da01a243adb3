"""The calls around a block together, as residual.py runs them: gradients of a whole network against those of its formula in
float64.

Bounds. A gradient passes through at most 12 roundings to bfloat16 a block (v, z, a, y, the gate's product, dy, dgate, dz, dv
and the weights' copies twice over) and two at the classifier, each off by at most half a step, 2^-8, of its value. They are
independent, so a tensor's error in the 2-norm grows with the root of their number: 2 sqrt(12 L + 2) 2^-8 of the tensor's
norm, the factor 2 for the products' and norms' gain. The classifier's gradient is a TF32 product (2^-10) of the same
activations. The global norm is a root of sums and keeps the relative error.
"""

import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def R():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_1905_07931_gb300 import csrtrain, residual
    csrtrain.lib()
    return residual


def _net(R, **kw):
    net = R.ResidualNet(200, 136, 2, 10, 72, seed=1, r_scale=0.9 if kw.get("norm") else 1.0, **kw)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(2)
    if net.vocab is not None:
        net.tokens.copy_((torch.rand(72, generator=gen, device="cuda") ** 3 * net.vocab).int())
        net.tokens[5] = -1   # a padded column
    else:
        net.x[0].copy_(torch.randn(200, 72, generator=gen, device="cuda"))
    net.labels.copy_(torch.randint(0, 10, (72,), generator=gen, device="cuda"))
    if net.norm is not None:
        net.wn.add_(0.2 * torch.randn(net.wn.shape, generator=gen, device="cuda"))
        net.bn.add_(0.2 * torch.randn(net.bn.shape, generator=gen, device="cuda"))
    net.b1.add_(0.1 * torch.randn(net.b1.shape, generator=gen, device="cuda"))
    net.b2.add_(0.1 * torch.randn(net.b2.shape, generator=gen, device="cuda"))
    return net


def _reference(net):
    """Loss and gradients in float64, from the weights' 16-bit copies."""
    p = {"w1": net.w1h, "w2": net.w2h, "b1": net.b1, "b2": net.b2}
    if net.norm is not None:
        p.update(wn=net.wn, bn=net.bn)
    if net.gate is not None:
        p["wg"] = net.wgh
    if net.vocab is not None:
        p["table"] = net.table
    wc = torch.zeros(net.classes, net.d, dtype=torch.float64)
    (rp, ci, val), _ = net.wc[net.cur].to_host()
    for i in range(net.classes):
        wc[i, ci[rp[i]:rp[i + 1]]] = torch.from_numpy(val[rp[i]:rp[i + 1]]).double()
    p["wc"] = wc.cuda()
    p = {k: v.double().clone().requires_grad_() for k, v in p.items()}

    def norm(x, k):
        if net.norm == "layer":
            x = x - x.mean(0)
        return x / (x.square().mean(0) + 1e-5).sqrt() * p["wn"][k][:, None] + p["bn"][k][:, None]

    def gelu(z):
        return 0.5 * z * (1 + torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)))

    if net.vocab is not None:
        h = math.sqrt(net.d) * p["table"][net.tokens.long().clamp_min(0)].t() * (net.tokens >= 0)
    else:
        h = net.x[0].double()
    for i in range(net.L):
        v = norm(h, i) if net.norm is not None else h
        y = p["w2"][i] @ gelu(p["w1"][i] @ v + p["b1"][i][:, None]) + p["b2"][i][:, None]
        if net.norm is not None:
            y = norm(y, net.L + 1 + i)
        if net.gate is not None:
            g = p["wg"][i] @ v
            s = torch.sigmoid(g)
            y = y * {"none": g, "sigmoid": s, "silu": g * s}[net.gate]
        h = net.r_scale * h + y
    out = norm(h, net.L) if net.norm is not None else h
    loss = torch.nn.functional.cross_entropy((p["wc"] @ out).t() + net.bc.double(), net.labels.long())
    loss.backward()
    return float(loss.detach()), {k: v.grad for k, v in p.items()}


CASES = [dict(norm="rms", gate="silu", vocab=90), dict(norm="layer", gate="sigmoid"), dict(norm="layer", vocab=90),
         dict(norm="rms", gate="none"), dict(vocab=90), dict()]


@pytest.mark.parametrize("kw", CASES, ids=lambda k: "-".join(f"{a}={b}" for a, b in k.items()) or "plain")
def test_gradients(R, kw):
    net = _net(R, **kw)
    loss, want = _reference(net)
    net.forward()
    R.C.softmax_xent(net.logits, net.labels, net.dlogits, net.loss)
    net.backward()
    tol = 2 * math.sqrt(12 * net.L + 2) * 2.0 ** -8
    assert abs(float(net.loss[0]) - loss) <= tol * loss
    got = {"w1": net.g1, "w2": net.g2, "b1": net.db1, "b2": net.db2, "wc": net.gc}
    if net.norm is not None:
        got.update(wn=net.dwn, bn=net.dbn)
    if net.gate is not None:
        got["wg"] = net.gg
    if net.vocab is not None:
        got["table"] = net.dtable
    for k, g in got.items():
        w = want[k]
        assert float((g.double() - w).norm()) <= tol * float(w.norm()), (k, float((g.double() - w).norm() / w.norm()))
    assert net.status() == 0


@pytest.mark.parametrize("kw", [dict(norm="rms", gate="silu", vocab=90, clip=0.05), dict(clip=0.05), dict(norm="layer", clip=1e6)],
                         ids=["all", "plain", "inactive"])
def test_clipped_step(R, kw):
    """A step's global norm is that of the formula's gradients, and what the updates see is scaled to the limit."""
    net = _net(R, **kw)
    _, want = _reference(net)
    total = math.sqrt(sum(float(w.square().sum()) for w in want.values()))
    tol = 2 * math.sqrt(12 * net.L + 2) * 2.0 ** -8
    net.step(0.003, 0.1)
    norm, factor = net.grad_norm.tolist()
    assert abs(norm - total) <= tol * total
    assert abs(factor - min(1.0, kw["clip"] / norm)) <= 1e-6 * factor
    after = math.sqrt(sum(float(g.double().square().sum()) for g in net.grads))
    assert abs(after - factor * norm) <= 1e-5 * after
    assert net.status() == 0
    net.step(0.003, 0.1)   # and goes on
    assert math.isfinite(float(net.loss[0])) and net.status() == 0


def test_command_runs(R, capsys):
    R.main(["--features", "96", "--hidden", "64", "--blocks", "2", "--batch", "40", "--steps", "2", "--norm", "rms", "--gate", "silu",
            "--vocab", "50", "--clip", "1"])
    assert '"grad_norm"' in capsys.readouterr().out


def test_two_streams_at_once(R):
    """Every call on two streams with a workspace each, many times over: the results are those of the calls one by one."""
    C = R.C
    gen = torch.Generator(device="cuda")
    gen.manual_seed(11)

    def work(k):
        d, n, vocab = 1040 + 8 * k, 1500 + 5 * k, 700
        s = {"y": torch.randn(d, n, generator=gen, device="cuda").bfloat16(), "r": torch.randn(d, n, generator=gen, device="cuda"),
             "g": torch.randn(d, n, generator=gen, device="cuda").bfloat16(),
             "tok": torch.randint(-1, vocab, (n,), generator=gen, device="cuda").int(),
             "table": torch.randn(vocab, d, generator=gen, device="cuda")}
        s["h"], s["v"], s["x"] = torch.empty_like(s["r"]), torch.empty_like(s["y"]), torch.empty_like(s["y"])
        s["dr"], s["dy"], s["dg"], s["dt"] = (torch.empty_like(s[q]) for q in ("r", "y", "g", "table"))
        stat = [torch.empty(n, device="cuda") for _ in range(4)]
        s["dw"] = [torch.empty(d, device="cuda") for _ in range(4)]
        P = C.Norm("layer", mean=stat[0], rstd=stat[1], dweight=s["dw"][0], dbias=s["dw"][1])
        Q = C.Norm("rms", rstd=stat[2], dweight=s["dw"][2], dbias=s["dw"][3])
        wsn, wse, wsk = C.BlockNormWorkspace(d, n), C.EmbedWorkspace(vocab, d, n), C.GradWorkspace()
        small, out = [s["dw"][0], s["dw"][2]], [torch.empty(d, device="cuda") for _ in range(2)]
        s["out"], s["norm"] = out, torch.zeros(2, device="cuda")

        def run():
            C.embed_fwd(s["table"], s["tok"], s["x"], wse, scale=0.5)
            C.block_norm_fwd(s["y"], s["r"], s["h"], s["v"], post=P, pre=Q, gate=s["g"], gate_act="silu")
            C.block_norm_bwd(s["v"], s["r"], s["h"], s["y"], s["dr"], s["dy"], wsn, post=P, pre=Q, gate=s["g"], gate_act="silu",
                             dgate=s["dg"])
            C.embed_bwd(s["dy"], s["tok"], s["dt"], wse)
            C.grad_clip(small, 1e-3, s["norm"], wsk, out=out)

        return s, run, (wsn, wse, wsk)

    works = [work(k) for k in range(2)]
    names = ("h", "v", "x", "dr", "dy", "dg", "dt", "norm")
    want = []
    for s, run, _ in works:
        run()
        torch.cuda.synchronize()
        want.append([s[q].clone() for q in names] + [t.clone() for t in s["dw"] + s["out"]])
    streams = [torch.cuda.Stream() for _ in works]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    for _ in range(20):
        for stream, (s, run, _) in zip(streams, works):
            with torch.cuda.stream(stream):
                run()
    torch.cuda.synchronize()
    for (s, _, workspaces), w in zip(works, want):
        got = [s[q] for q in names] + s["dw"] + s["out"]
        assert all(torch.equal(a, b) for a, b in zip(got, w))
        assert all(ws.status()[0] == 0 for ws in workspaces)


def test_clipping_takes_the_classifiers_bias(R):
    """With small inputs most of the gradient is the classifier's bias's: the norm holds it, and its update is scaled with
    the others'."""
    net = _net(R, clip=0.01)
    net.x[0].mul_(1e-3)
    net.b1.zero_()
    net.b2.zero_()
    net.bc.copy_(torch.linspace(-2, 2, net.classes))
    before = net.bc.clone()
    net.bc.requires_grad_()
    _, want = _reference(net)
    bias = net.bc.grad.double()
    net.bc.requires_grad_(False)
    total = math.sqrt(sum(float(w.square().sum()) for w in want.values()) + float(bias.square().sum()))
    # without it the norm would be 1 - sqrt(1 - 0.5^2) = 13% smaller, or more: far outside tol, which is 4%
    assert float(bias.norm()) > 0.5 * total and total > 9 * net.clip
    tol = 2 * math.sqrt(12 * net.L + 2) * 2.0 ** -8
    net.step(0.003, 0.1)
    norm, factor = net.grad_norm.tolist()
    assert abs(norm - total) <= tol * total and abs(factor - net.clip / norm) <= 1e-6 * factor
    step = 0.003 * factor * bias
    assert ((net.bc.double() - (before.double() - step)).norm() <= 2 * tol * step.norm() + 2.0 ** -23 * before.double().norm())
    assert abs(math.sqrt(sum(float(g.double().square().sum()) for g in net.grads)) - net.clip) <= 1e-5 * net.clip
    assert net.status() == 0
