"""The dense layer's products and the orthogonalised update: cases, plain forms and work.

Layouts are the library's: weights W are M x K, activations are feature-major (X is K x n, Y is M x n, the token
index contiguous). Three kinds of case:

fwd   y = act(W x + b) + r, and the pre-activation z where a backward pass will want it. W, x, r, z and y are
      16-bit (bfloat16 or float16), b is float32.
bwd   a layer's backward pass from dy = dL/d(pre-activation): dx = (W^T dy) * act'(z_below) + r for the layer
      below (act' and r where the case has them), dW = dy x^T and db = the row sums of dy in float32.
muon  the momentum of a batch of gradients and its orthogonalised direction (Newton-Schulz):
      m <- beta m + g;  u = g + beta m;  X = u / max(||u||_F, eps);  5 times X <- a X + (b A + c A A) X with
      A = X X^T (X^T X on the right where X has more rows than columns);  o = scale X, in bfloat16.
"""

import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
ACTS = ("none", "relu", "gelu", "silu")
NS_A, NS_B, NS_C = 3.4445, -4.7750, 2.0315
BETA, EPS, STEPS = 0.95, 1e-7, 5


def listed():
    return [
        # serving: one token through a hidden layer of 4096 units
        dict(name="fwd one token", kind="fwd", m=4096, k=4096, n=1, dtype="bf16", act="gelu", bias=True, residual=False,
             z=False, pad=False),
        # serving: a few sequences decode together, in float16, back into the residual stream
        dict(name="fwd few tokens f16", kind="fwd", m=4096, k=9216, n=24, dtype="f16", act="none", bias=True,
             residual=True, z=False, pad=False),
        # training on ragged prompts: an odd number of tokens packed without padding, z kept for the backward pass
        dict(name="fwd ragged", kind="fwd", m=1000, k=4096, n=777, dtype="bf16", act="relu", bias=True, residual=False,
             z=True, pad=False),
        # training on long prompts: the largest forward product, everything in the epilogue
        dict(name="fwd prompt", kind="fwd", m=4096, k=4096, n=8192, dtype="bf16", act="gelu", bias=True, residual=True,
             z=True, pad=False),
        # the small classifier's first layer at its batch, in float16
        dict(name="bwd small f16", kind="bwd", m=300, k=784, n=256, dtype="f16", act="relu", residual=False, pad=False),
        # the wide head's first layer at its batch: no layer below
        dict(name="bwd head", kind="bwd", m=4096, k=9216, n=256, dtype="bf16", act="none", residual=False, pad=False),
        # a ragged batch in a wider buffer (strided rows)
        dict(name="bwd ragged", kind="bwd", m=1000, k=4096, n=1777, dtype="bf16", act="silu", residual=False, pad=True),
        # training on long prompts: the largest backward pass, act' and the residual's gradient in the epilogue
        dict(name="bwd prompt", kind="bwd", m=4096, k=4096, n=8192, dtype="bf16", act="gelu", residual=True, pad=False),
        # one update of the small classifier's first layer
        dict(name="muon small", kind="muon", batch=1, m=300, k=784, dtype="f32"),
        # the layers of one shape of a stack of blocks, updated together, gradients in bfloat16
        dict(name="muon blocks", kind="muon", batch=12, m=512, k=2048, dtype="bf16"),
        # a tall matrix (more outputs than inputs), sizes no power of two
        dict(name="muon tall", kind="muon", batch=1, m=4096, k=1000, dtype="f32"),
        # the wide head's first layer, the largest update
        dict(name="muon head", kind="muon", batch=1, m=4096, k=9216, dtype="f32"),
    ]


def _log(rng, lo, hi):
    """A size between lo and hi, even over its logarithm, half of them multiples of 8, the rest as they come."""
    v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    if rng.random() < 0.5:
        v = (v + 7) // 8 * 8
    v = min(max(v, lo), hi)
    return v + 8 if v == 3072 else v


def draw(rng):
    kind = rng.choice(("fwd", "fwd", "bwd", "muon"))
    while True:
        if kind == "muon":
            c = dict(kind=kind, batch=rng.choice((1, 1, 2, 3, 6, 12)), m=_log(rng, 64, 4096), k=_log(rng, 64, 9216),
                     dtype=rng.choice(("f32", "bf16")))
            s, l = min(c["m"], c["k"]), max(c["m"], c["k"])
            if c["batch"] * s * s * (2 * l + s) <= 4096 * 4096 * (2 * 9216 + 4096):
                return c
            continue
        c = dict(kind=kind, m=_log(rng, 64, 9216), k=_log(rng, 64, 9216), n=_log(rng, 1 if kind == "fwd" else 16, 8192),
                 dtype=rng.choice(("bf16", "f16")), act=rng.choice(ACTS))
        if kind == "fwd":
            c["bias"] = rng.random() < 0.7
        c["residual"] = rng.random() < 0.5
        if kind == "fwd":
            c["z"] = rng.random() < 0.5
        c["pad"] = rng.random() < 0.3
        if c["m"] * c["k"] * c["n"] <= 4096 * 4096 * 8192:
            return c


def _columns(rows, n, dtype, pad, gen, scale=1.0):
    """rows x n activations; with pad, columns of a buffer whose rows are wider (a multiple of 64 tokens)."""
    wide = (n + 63) // 64 * 64 if pad else n
    t = torch.randn(rows, wide, generator=gen, device="cuda").mul_(scale).to(dtype)
    return t[:, :n]


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    s = dict(case)
    dt = DTYPES[case["dtype"]]
    if case["kind"] == "muon":
        b, m, k = case["batch"], case["m"], case["k"]
        # gradients as training gives them: a few strong directions over noise; momentum of some steps before
        r = 8
        strong = torch.randn(b, m, r, generator=gen, device="cuda") @ torch.randn(b, r, k, generator=gen, device="cuda")
        s["g"] = (1e-3 * (torch.randn(b, m, k, generator=gen, device="cuda") + 0.2 * strong)).to(dt)
        s["mom"] = 3e-3 * (torch.randn(b, m, k, generator=gen, device="cuda") + 0.5 * strong)
        s["o"] = torch.empty(b, m, k, dtype=torch.bfloat16, device="cuda")
        s["scale"] = 0.2 * math.sqrt(max(m, k))
        if own:
            from paper_1905_07931_gb300 import csrtrain as C
            s["ws"] = C.OrthogonalizeWorkspace(b, m, k)
        return s
    m, k, n, pad = case["m"], case["k"], case["n"], case["pad"]
    s["w"] = (torch.randn(m, k, generator=gen, device="cuda") / math.sqrt(k)).to(dt)
    s["x"] = _columns(k, n, dt, pad, gen)
    if case["kind"] == "fwd":
        s["b"] = 0.1 * torch.randn(m, generator=gen, device="cuda") if case["bias"] else None
        s["r"] = _columns(m, n, dt, pad, gen) if case["residual"] else None
        s["y"] = torch.empty(m, n, dtype=dt, device="cuda")
        s["z_out"] = torch.empty(m, n, dtype=dt, device="cuda") if case["z"] else None
    else:
        s["dy"] = _columns(m, n, dt, pad, gen, 0.05)
        s["z_below"] = _columns(k, n, dt, pad, gen) if case["act"] != "none" else None
        s["r"] = _columns(k, n, dt, pad, gen, 0.05) if case["residual"] else None
        s["dx"] = torch.empty(k, n, dtype=dt, device="cuda")
        s["dw"] = torch.empty(m, k, dtype=torch.float32, device="cuda")
        s["db"] = torch.empty(m, dtype=torch.float32, device="cuda")
    if own:
        from paper_1905_07931_gb300 import csrtrain as C
        s["ws"] = C.DenseWorkspace(m, k, n)
    return s


def _act(z, act):
    if act == "relu":
        return torch.where(z > 0, z, torch.zeros_like(z))
    if act == "gelu":
        return 0.5 * z * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (z + 0.044715 * z * z * z)))
    if act == "silu":
        return z / (1.0 + torch.exp(-z))
    return z


def _act_grad(z, act):
    if act == "relu":
        return (z > 0).to(z.dtype)
    if act == "gelu":
        t = torch.tanh(math.sqrt(2.0 / math.pi) * (z + 0.044715 * z * z * z))
        return 0.5 * (1.0 + t) + 0.5 * z * (1.0 - t * t) * math.sqrt(2.0 / math.pi) * (1.0 + 3 * 0.044715 * z * z)
    if act == "silu":
        p = 1.0 / (1.0 + torch.exp(-z))
        return p * (1.0 + z * (1.0 - p))
    return torch.ones_like(z)


def _plain_muon(s):
    g, mom = s["g"].float(), s["mom"]
    mom.mul_(BETA).add_(g)
    x = g + BETA * mom
    x = x / x.square().sum(dim=(1, 2), keepdim=True).sqrt().clamp_min(EPS)
    tall = s["m"] > s["k"]
    x = x.transpose(1, 2) if tall else x
    for _ in range(STEPS):
        a = x @ x.transpose(1, 2)
        x = NS_A * x + (NS_B * a + NS_C * (a @ a)) @ x
    x = x.transpose(1, 2) if tall else x
    return (s["scale"] * x).to(torch.bfloat16), mom


def run(s):
    if own:
        from paper_1905_07931_gb300 import csrtrain as C
        if s["kind"] == "fwd":
            C.dense_fwd(s["w"], s["x"], s["y"], s["ws"], bias=s["b"], act=s["act"], residual=s["r"], z=s["z_out"])
            return {"y": s["y"], "z": s["z_out"]}
        if s["kind"] == "bwd":
            C.dense_bwd_x(s["w"], s["dy"], s["dx"], s["ws"], z_below=s["z_below"], act=s["act"], residual=s["r"])
            C.dense_bwd_w(s["dy"], s["x"], s["dw"], s["ws"], db=s["db"])
            return {"dx": s["dx"], "dw": s["dw"], "db": s["db"]}
        C.orthogonalize(s["g"], s["o"], s["ws"], momentum=s["mom"], beta=BETA, nesterov=True, steps=STEPS, eps=EPS,
                        scale=s["scale"])
        return {"o": s["o"], "mom": s["mom"]}
    if s["kind"] == "muon":
        o, mom = _plain_muon(s)
        return {"o": o, "mom": mom}
    w, dt = s["w"].float(), s["w"].dtype
    if s["kind"] == "fwd":
        z = w @ s["x"].float()
        if s["b"] is not None:
            z = z + s["b"][:, None]
        y = _act(z, s["act"])
        if s["r"] is not None:
            y = y + s["r"].float()
        return {"y": y.to(dt), "z": z.to(dt) if s["z_out"] is not None else None}
    dy = s["dy"].float()
    dx = w.t() @ dy
    if s["z_below"] is not None:
        dx = dx * _act_grad(s["z_below"].float(), s["act"])
    if s["r"] is not None:
        dx = dx + s["r"].float()
    return {"dx": dx.to(dt), "dw": dy @ s["x"].float().t(), "db": dy.sum(dim=1)}


def work(case):
    m, k = case["m"], case["k"]
    if case["kind"] == "muon":
        b, s, l = case["batch"], min(m, k), max(m, k)
        size = 4 if case["dtype"] == "f32" else 2
        # A and A A are symmetric: half of their products are enough
        return {"bytes": b * m * k * (size + 4 + 4 + 2), "flops": b * STEPS * (s * (s + 1) * l + s * s * (s + 1) + 2 * s * s * l)}
    n = case["n"]
    if case["kind"] == "fwd":
        cells = m * k + k * n + m * n * (1 + case["residual"] + case["z"])
        return {"bytes": 2 * cells + 4 * m * case["bias"], "flops": 2 * m * k * n}
    cells = m * k + m * n + k * n * (2 + (case["act"] != "none") + case["residual"])
    return {"bytes": 2 * cells + 4 * m * k + 4 * m, "flops": 4 * m * k * n}


def _sigmoid64(v):
    return 0.5 * (1.0 + torch.tanh(0.5 * v))


def exact(case, seed):
    """From the definitions in 64 bits: the gelu and its derivative through the sigmoid, the products as sums."""
    s = prepare(case, seed)
    if case["kind"] == "muon":
        g, mom = s["g"].double(), s["mom"].double()
        mom = BETA * mom + g
        u = g + BETA * mom
        out = torch.empty_like(u)
        for i in range(case["batch"]):
            x = u[i] / max(float(torch.linalg.matrix_norm(u[i])), EPS)
            eye = torch.eye(min(case["m"], case["k"]), dtype=torch.float64, device=x.device)
            for _ in range(STEPS):
                if case["m"] > case["k"]:
                    a = torch.mm(x.t(), x)
                    x = torch.mm(x, NS_A * eye + NS_B * a + NS_C * torch.mm(a, a))
                else:
                    a = torch.mm(x, x.t())
                    x = torch.mm(NS_A * eye + NS_B * a + NS_C * torch.mm(a, a), x)
            out[i] = s["scale"] * x
        return {"o": out, "mom": mom}
    w, x = s["w"].double(), s["x"].double()
    root = math.sqrt(2.0 / math.pi)
    if case["kind"] == "fwd":
        z = torch.einsum("mk,kn->mn", w, x)
        if s["b"] is not None:
            z = z + s["b"].double().unsqueeze(1)
        gate = {"none": 1.0, "relu": (z > 0).double(), "silu": _sigmoid64(z),
                "gelu": _sigmoid64(2.0 * root * (z + 0.044715 * z.pow(3)))}[case["act"]]
        y = z * gate
        if s["r"] is not None:
            y = y + s["r"].double()
        return {"y": y, "z": z if case["z"] else None}
    dy = s["dy"].double()
    dx = torch.einsum("mk,mn->kn", w, dy)
    if s["z_below"] is not None:
        z = s["z_below"].double()
        if case["act"] == "relu":
            dx = torch.where(z > 0, dx, torch.zeros_like(dx))
        else:
            v, dv = (z, 1.0) if case["act"] == "silu" else (
                2.0 * root * (z + 0.044715 * z.pow(3)), 2.0 * root * (1.0 + 0.134145 * z.pow(2)))
            p = _sigmoid64(v)
            dx = dx * (p + z * p * (1.0 - p) * dv)
    if s["r"] is not None:
        dx = dx + s["r"].double()
    return {"dx": dx, "dw": torch.einsum("mn,kn->mk", dy, x), "db": dy.sum(dim=1)}
