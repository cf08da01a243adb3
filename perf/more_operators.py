"""Operators around the dense products of a residual network over tokens: cases, plain forms and work.

Layouts are the library's: activations are feature-major (d x n, the token index contiguous). Five kinds of case:

norm_fwd   between two blocks: the norm after a block, its gate, the scaled residual and the norm before the next:
           t = N_post(y);  h = r_scale r + a(g) t;  v = N_pre(h), N one of
             rms    x / sqrt(mean(x^2) + eps) * weight
             layer  (x - mean(x)) / sqrt(var(x) + eps) * weight + bias
             scale  x * weight                                          (after a block only)
           over the d features of each token; a(g) none (h = r_scale r + t), g, sigmoid(g) or silu(g). The means and
           reciprocal deviations are kept for the backward pass.
norm_bwd   its backward pass from dv and dh: gradients of r, y, g, the weights and the biases.
embed_fwd  x[:, c] = scale table[token c, :].
embed_bwd  dtable[v, :] = (dtable[v, :] +) scale times the sum of dx[:, c] over the tokens c that are v.
clip       norm = sqrt of the sum of squares over all gradients; out = g min(1, max_norm / norm), into the
           optimiser's buffers.
"""

import math
import random

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
SIZE = {"bf16": 2, "f16": 2, "f32": 4}
EPS = 1e-5
MOST = 4096 * 8192   # largest d x n


def listed():
    return [
        # serving: one token on its way between two blocks of 4096 features
        dict(name="norm fwd one token", kind="norm_fwd", d=4096, n=1, dtype="bf16", stream="bf16", post="rms", pre="rms",
             gate="off", bias=False, pad=False),
        # ragged prompts packed without padding, an odd number of tokens, float16, a gated block between layer norms
        dict(name="norm fwd ragged f16", kind="norm_fwd", d=1000, n=777, dtype="f16", stream="f16", post="layer",
             pre="layer", gate="silu", bias=True, pad=False),
        # training on long prompts: the largest forward pass
        dict(name="norm fwd prompt", kind="norm_fwd", d=4096, n=8192, dtype="bf16", stream="bf16", post="rms", pre="rms",
             gate="sigmoid", bias=False, pad=False),
        # the residual network at its batch
        dict(name="norm bwd small", kind="norm_bwd", d=784, n=256, dtype="bf16", stream="bf16", post="scale", pre="layer",
             gate="off", bias=True, pad=False),
        # a ragged batch in a wider buffer, the residual stream in float32
        dict(name="norm bwd ragged", kind="norm_bwd", d=4096, n=1777, dtype="bf16", stream="f32", post="layer",
             pre="layer", gate="plain", bias=True, pad=True),
        # training on long prompts: the largest backward pass
        dict(name="norm bwd prompt", kind="norm_bwd", d=4096, n=8192, dtype="bf16", stream="bf16", post="rms", pre="rms",
             gate="sigmoid", bias=False, pad=False),
        # serving: a few sequences' next tokens
        dict(name="embed fwd few tokens", kind="embed_fwd", vocab=10000, d=4096, n=24, table="bf16", dtype="bf16"),
        # training on long prompts, float32 master table into 16-bit activations
        dict(name="embed fwd prompt", kind="embed_fwd", vocab=32768, d=4096, n=8192, table="f32", dtype="bf16"),
        # a ragged batch, added to what a classifier that shares the table has left there
        dict(name="embed bwd ragged tied", kind="embed_bwd", vocab=10000, d=1000, n=777, table="f32", dtype="f16",
             accumulate=True),
        # training on long prompts: the whole gradient of the largest table
        dict(name="embed bwd prompt", kind="embed_bwd", vocab=32768, d=4096, n=8192, table="f32", dtype="bf16",
             accumulate=False),
        # all gradients of the residual network: its matrices, biases and norm weights
        dict(name="clip residual network", kind="clip", form="blocks", blocks=3, d=784, h=1024, dtype="f32", out="f32"),
        # all gradients of the wide head (9216-4096-4096-1000)
        dict(name="clip wide head", kind="clip", form="head", dtype="f32", out="f32"),
    ]


def _log(rng, lo, hi):
    """A size between lo and hi, even over its logarithm, half of them multiples of 8, the rest as they come."""
    v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    if rng.random() < 0.5:
        v = (v + 7) // 8 * 8
    return min(max(v, lo), hi)


def draw(rng):
    kind = rng.choice(("norm_fwd", "norm_fwd", "norm_bwd", "norm_bwd", "embed_fwd", "embed_bwd", "clip"))
    while True:
        if kind in ("norm_fwd", "norm_bwd"):
            dt = rng.choice(("bf16", "f16"))
            c = dict(kind=kind, d=_log(rng, 64, 9216), n=_log(rng, 1, 8192), dtype=dt,
                     stream=rng.choice((dt, dt, "f32")), post=rng.choice(("rms", "layer", "scale")),
                     pre=rng.choice(("rms", "layer")), gate=rng.choice(("off", "plain", "sigmoid", "silu")),
                     bias=rng.random() < 0.5, pad=rng.random() < 0.3)
            # bytes of the largest listed pass of the direction
            if c["d"] * c["n"] * (1 if c["stream"] != "f32" else 1.6) <= MOST:
                return c
        elif kind == "clip":
            c = dict(kind=kind, form="mixed", count=_log(rng, 1, 60), smallest=_log(rng, 1, 1000),
                     largest=_log(rng, 1000, 4096 * 4096), sizes=rng.randrange(1 << 20), active=rng.random() < 0.8,
                     dtype=rng.choice(("f32", "bf16")), out=rng.choice(("f32", "f32", "bf16")))
            if sum(r * k for r, k in _shapes(c)) <= 4096 * (9216 + 4096):
                return c
        else:
            c = dict(kind=kind, vocab=_log(rng, 100, 65536), d=_log(rng, 64, 4096), n=_log(rng, 1, 8192),
                     table=rng.choice(("f32", "f32", "bf16")), dtype=rng.choice(("bf16", "f16")))
            if kind == "embed_bwd":
                c["accumulate"] = rng.random() < 0.4
            if c["vocab"] * c["d"] <= 32768 * 4096:
                return c


def _shapes(case):
    """The gradients of a clip case, as rows and columns."""
    if case["form"] == "blocks":
        d, h = case["d"], case["h"]
        one = [(h, d), (1, h), (d, h), (1, d), (1, d), (1, d)]
        return one * case["blocks"]
    if case["form"] == "head":
        return [(4096, 9216), (1, 4096), (4096, 4096), (1, 4096), (1000, 4096), (1, 1000)]
    rng = random.Random(case["sizes"])
    lo, hi = math.log(case["smallest"]), math.log(max(case["largest"], case["smallest"]))
    return [(1, int(round(math.exp(rng.uniform(lo, hi))))) for _ in range(case["count"])]


def _columns(rows, n, dtype, pad, gen, scale=1.0):
    """rows x n activations; with pad, columns of a buffer whose rows are wider (a multiple of 64 tokens)."""
    wide = (n + 63) // 64 * 64 if pad else n
    t = torch.randn(rows, wide, generator=gen, device="cuda").mul_(scale).to(dtype)
    return t[:, :n]


def _zipf(vocab):
    """How often each token comes: as in text, the v-th most frequent with 1 / (v + 2.7), over shuffled numbers."""
    return 1.0 / (torch.arange(vocab, dtype=torch.float64) + 2.7)


def _tokens(vocab, n, gen):
    p = _zipf(vocab).cuda().cumsum(0)
    rank = torch.searchsorted(p, torch.rand(n, generator=gen, device="cuda", dtype=torch.float64) * p[-1])
    return torch.randperm(vocab, generator=gen, device="cuda")[rank.clamp_max(vocab - 1)].to(torch.int32)


def _distinct(vocab, n):
    """How many different tokens n of them are expected to hold."""
    p = _zipf(vocab)
    return float((1.0 - (1.0 - p / p.sum()) ** n).sum())


def _vector(d, gen, around):
    return around + 0.1 * torch.randn(d, generator=gen, device="cuda")


def _statistics(x, kind):
    """Mean and reciprocal deviation of each token's features."""
    if kind == "scale":
        return None, None
    x = x.double()
    mean = x.mean(0) if kind == "layer" else torch.zeros_like(x[0])
    rstd = ((x - mean).square().mean(0) + EPS).rsqrt()
    return (mean.float() if kind == "layer" else None), rstd.float()


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    s = dict(case)
    kind = case["kind"]
    if kind == "clip":
        s["g"] = [(torch.randn(shape, generator=gen, device="cuda") * 10.0 ** (-3 + i % 3)).to(DTYPES[case["dtype"]])
                  for i, shape in enumerate(_shapes(case))]
        s["into"] = [torch.empty(g.shape, dtype=DTYPES[case["out"]], device="cuda") for g in s["g"]]
        # below the norm, so that the gradients are scaled; in some drawn cases they are small enough to pass as they are
        s["max_norm"] = (3e-4 if case.get("active", True) else 1.0) * math.sqrt(sum(g.numel() for g in s["g"]))
        s["norm"] = torch.zeros(2, device="cuda")
        if own:
            from paper_1905_07931_gb300 import csrtrain as C
            s["ws"] = C.GradWorkspace()
            s["glist"], s["olist"] = C.TensorList(s["g"]), C.TensorList(s["into"])
        return s
    d, n, dt = case["d"], case["n"], DTYPES[case["dtype"]]
    if kind in ("embed_fwd", "embed_bwd"):
        vocab, tt = case["vocab"], DTYPES[case["table"]]
        s["tokens"] = _tokens(vocab, n, gen)
        s["scale"] = math.sqrt(d)
        if kind == "embed_fwd":
            s["w"] = (torch.randn(vocab, d, generator=gen, device="cuda") / math.sqrt(d)).to(tt)
            s["x"] = torch.empty(d, n, dtype=dt, device="cuda")
        else:
            s["dx"] = _columns(d, n, dt, False, gen, 0.05)
            s["dw"] = torch.randn(vocab, d, generator=gen, device="cuda").mul_(0.05).to(tt)
        if own:
            from paper_1905_07931_gb300 import csrtrain as C
            s["ws"] = C.EmbedWorkspace(vocab, d, n)
        return s
    st, pad = DTYPES[case["stream"]], case["pad"]
    s["scale_r"] = 0.9
    s["wpost"], s["wpre"] = _vector(d, gen, 1.0), _vector(d, gen, 1.0)
    s["bpost"] = _vector(d, gen, 0.0) if case["bias"] and case["post"] != "rms" else None
    s["bpre"] = _vector(d, gen, 0.0) if case["bias"] and case["pre"] == "layer" else None
    # a block's output with tokens of different size and an offset; the stream that many blocks have added to
    size = torch.exp(torch.randn(n, generator=gen, device="cuda"))
    s["y"] = _columns(d, n, dt, pad, gen, 0.7)
    s["y"].mul_(size.to(dt)).add_((0.3 * size).to(dt))
    s["g"] = _columns(d, n, dt, pad, gen) if case["gate"] != "off" else None
    if kind == "norm_fwd":
        s["r"] = _columns(d, n, st, pad, gen, 3.0)
        s["h"] = torch.empty(d, n, dtype=st, device="cuda")
        s["v"] = torch.empty(d, n, dtype=dt, device="cuda")
        s["mpost"] = torch.empty(n, device="cuda") if case["post"] == "layer" else None
        s["spost"] = torch.empty(n, device="cuda") if case["post"] != "scale" else None
        s["mpre"] = torch.empty(n, device="cuda") if case["pre"] == "layer" else None
        s["spre"] = torch.empty(n, device="cuda")
    else:
        s["h"] = _columns(d, n, st, pad, gen, 3.0)
        s["dv"] = _columns(d, n, dt, pad, gen, 0.05)
        s["dh"] = _columns(d, n, st, pad, gen, 0.05)
        s["mpost"], s["spost"] = _statistics(s["y"], case["post"])
        s["mpre"], s["spre"] = _statistics(s["h"], case["pre"])
        s["dr"] = torch.empty(d, n, dtype=st, device="cuda")
        s["dy"] = torch.empty(d, n, dtype=dt, device="cuda")
        s["dg"] = torch.empty(d, n, dtype=dt, device="cuda") if s["g"] is not None else None
        for side in ("post", "pre"):
            s["dw" + side] = torch.empty(d, device="cuda")
            s["db" + side] = torch.empty(d, device="cuda") if s["b" + side] is not None else None
    if own:
        from paper_1905_07931_gb300 import csrtrain as C
        for side in ("post", "pre"):
            s[side + "_norm"] = C.Norm(case[side], weight=s["w" + side], bias=s["b" + side], eps=EPS,
                                       mean=s["m" + side], rstd=s["s" + side], dweight=s.get("dw" + side),
                                       dbias=s.get("db" + side))
        if kind == "norm_bwd":
            s["ws"] = C.BlockNormWorkspace(d, n)
    return s


GATES = {"off": "none", "plain": "none", "sigmoid": "sigmoid", "silu": "silu"}


def _norm(x, kind, weight, bias):
    mean = rstd = None
    if kind == "layer":
        mean = x.mean(0)
        x = x - mean
    if kind != "scale":
        rstd = 1.0 / torch.sqrt((x * x).mean(0) + EPS)
        x = x * rstd
    x = x * weight[:, None]
    return (x if bias is None else x + bias[:, None]), mean, rstd


def _hat(x, mean, rstd):
    if mean is not None:
        x = x - mean
    return x if rstd is None else x * rstd


def _norm_grad(dout, hat, rstd, kind, weight):
    """Gradient of a norm's input, and of its weight and bias."""
    s = dout * weight[:, None]
    if kind != "scale":
        s = s - hat * (s * hat).mean(0) - (s.mean(0) if kind == "layer" else 0.0)
        s = s * rstd
    return s, (dout * hat).sum(1), dout.sum(1)


def _gate(g, gate):
    if gate == "plain":
        return g, torch.ones_like(g)
    p = 1.0 / (1.0 + torch.exp(-g))
    if gate == "sigmoid":
        return p, p * (1.0 - p)
    return g * p, p * (1.0 + g * (1.0 - p))


def run(s):
    if own:
        from paper_1905_07931_gb300 import csrtrain as C
    kind = s["kind"]
    if kind == "norm_fwd":
        if own:
            C.block_norm_fwd(s["y"], s["r"], s["h"], s["v"], post=s["post_norm"], pre=s["pre_norm"], gate=s["g"],
                             gate_act=GATES[s["gate"]], r_scale=s["scale_r"])
            return {k: s[k] for k in ("h", "v", "mpost", "spost", "mpre", "spre")}
        t, mpost, spost = _norm(s["y"].float(), s["post"], s["wpost"], s["bpost"])
        if s["g"] is not None:
            t = t * _gate(s["g"].float(), s["gate"])[0]
        h = s["scale_r"] * s["r"].float() + t
        v, mpre, spre = _norm(h, s["pre"], s["wpre"], s["bpre"])
        return {"h": h.to(s["h"].dtype), "v": v.to(s["v"].dtype), "mpost": mpost, "spost": spost, "mpre": mpre,
                "spre": spre}
    if kind == "norm_bwd":
        if own:
            C.block_norm_bwd(s["dv"], s["dh"], s["h"], s["y"], s["dr"], s["dy"], s["ws"], post=s["post_norm"],
                             pre=s["pre_norm"], gate=s["g"], gate_act=GATES[s["gate"]], dgate=s["dg"],
                             r_scale=s["scale_r"])
            return {k: s[k] for k in ("dr", "dy", "dg", "dwpost", "dbpost", "dwpre", "dbpre")}
        hat = _hat(s["h"].float(), s["mpre"], s["spre"])
        dh, dwpre, dbpre = _norm_grad(s["dv"].float(), hat, s["spre"], s["pre"], s["wpre"])
        dh = dh + s["dh"].float()
        hat = _hat(s["y"].float(), s["mpost"], s["spost"])
        dt, dg = dh, None
        if s["g"] is not None:
            a, slope = _gate(s["g"].float(), s["gate"])
            t = hat * s["wpost"][:, None]
            if s["bpost"] is not None:
                t = t + s["bpost"][:, None]
            dg = (dh * t * slope).to(s["dg"].dtype)
            dt = dh * a
        dy, dwpost, dbpost = _norm_grad(dt, hat, s["spost"], s["post"], s["wpost"])
        return {"dr": (s["scale_r"] * dh).to(s["dr"].dtype), "dy": dy.to(s["dy"].dtype), "dg": dg, "dwpost": dwpost,
                "dbpost": dbpost if s["bpost"] is not None else None, "dwpre": dwpre,
                "dbpre": dbpre if s["bpre"] is not None else None}
    if kind == "embed_fwd":
        if own:
            C.embed_fwd(s["w"], s["tokens"], s["x"], s["ws"], scale=s["scale"])
            return s["x"]
        return (s["scale"] * s["w"][s["tokens"].long()].float()).t().contiguous().to(s["x"].dtype)
    if kind == "embed_bwd":
        if own:
            C.embed_bwd(s["dx"], s["tokens"], s["dw"], s["ws"], scale=s["scale"], accumulate=s["accumulate"])
            return s["dw"]
        total = s["dw"].float() if s["accumulate"] else torch.zeros(s["dw"].shape, device="cuda")
        total.index_add_(0, s["tokens"].long(), s["scale"] * s["dx"].float().t())
        return s["dw"].copy_(total)
    if own:
        C.grad_clip(s["glist"], s["max_norm"], s["norm"], s["ws"], out=s["olist"])
        return {"norm": s["norm"], "out": s["into"]}
    total = sum((g.double() * g.double()).sum() for g in s["g"]).sqrt()
    factor = torch.where(total > s["max_norm"], s["max_norm"] / total, torch.ones_like(total)).float()
    for g, o in zip(s["g"], s["into"]):
        o.copy_(g.float() * factor)
    return {"norm": torch.stack([total.float(), factor]), "out": s["into"]}


def work(case):
    kind = case["kind"]
    if kind == "clip":
        cells = sum(r * k for r, k in _shapes(case))
        return {"bytes": cells * (SIZE[case["dtype"]] + SIZE[case["out"]]) + 8, "flops": 3 * cells}
    d, n, b = case["d"], case["n"], SIZE[case["dtype"]]
    if kind == "embed_fwd":
        return {"bytes": _distinct(case["vocab"], n) * d * SIZE[case["table"]] + d * n * b + 4 * n, "flops": d * n}
    if kind == "embed_bwd":
        rows = 2 * _distinct(case["vocab"], n) if case["accumulate"] else case["vocab"]
        return {"bytes": rows * d * SIZE[case["table"]] + d * n * b + 4 * n, "flops": 2 * d * n}
    st, gated = SIZE[case["stream"]], case["gate"] != "off"
    vectors = 4 * d * (2 + (case["bias"] and case["post"] != "rms") + (case["bias"] and case["pre"] == "layer"))
    stats = 4 * n * ((case["post"] != "scale") + (case["post"] == "layer") + 1 + (case["pre"] == "layer"))
    if kind == "norm_fwd":
        return {"bytes": d * n * (2 * b + 2 * st + b * gated) + vectors + stats, "flops": d * n * (14 + 4 * gated)}
    return {"bytes": d * n * (3 * b + 3 * st + 2 * b * gated) + 2 * vectors + stats, "flops": d * n * (26 + 10 * gated)}


def _sigmoid64(v):
    return 0.5 * (1.0 + torch.tanh(0.5 * v))


def _normalised64(x, kind):
    if kind == "scale":
        return x, None, None
    mean = x.mean(dim=0, keepdim=True) if kind == "layer" else torch.zeros_like(x[:1])
    rstd = torch.rsqrt(torch.mean((x - mean) ** 2, dim=0, keepdim=True) + EPS)
    return (x - mean) * rstd, (mean[0] if kind == "layer" else None), rstd[0]


def _affine64(x, weight, bias):
    x = x * weight.double().unsqueeze(1)
    return x if bias is None else x + bias.double().unsqueeze(1)


def _input_grad64(dout, weight, hat, rstd, kind):
    """The projection of the weighted gradient off the normalised input (and off the ones), over the deviation."""
    u = dout * weight.double().unsqueeze(1)
    if kind == "scale":
        return u
    along = torch.einsum("dn,dn->n", u, hat) / u.shape[0]
    u = u - hat * along
    if kind == "layer":
        ones = torch.mean(dout * weight.double().unsqueeze(1), dim=0)
        u = u - ones.unsqueeze(0)
    return u * rstd.double()


def exact(case, seed):
    """From the definitions in 64 bits."""
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "clip":
        norm = math.sqrt(sum(float(torch.linalg.vector_norm(g.double())) ** 2 for g in s["g"]))
        factor = min(1.0, s["max_norm"] / norm) if norm > 0 else 1.0
        return {"norm": torch.tensor([norm, factor], dtype=torch.float64, device="cuda"),
                "out": [g.double() * factor for g in s["g"]]}
    if kind == "embed_fwd":
        return s["scale"] * torch.index_select(s["w"], 0, s["tokens"].long()).double().transpose(0, 1)
    if kind == "embed_bwd":
        out = s["dw"].double() if case["accumulate"] else torch.zeros(s["dw"].shape, dtype=torch.float64, device="cuda")
        values, place = torch.unique(s["tokens"].long(), return_inverse=True)
        part = torch.zeros(len(values), case["d"], dtype=torch.float64, device="cuda")
        part.index_add_(0, place, s["dx"].double().transpose(0, 1))
        out[values] += s["scale"] * part
        return out
    g = None if s["g"] is None else s["g"].double()
    p = None if g is None else _sigmoid64(g)
    gate = {"off": 1.0, "plain": g, "sigmoid": p, "silu": None if g is None else g * p}[case["gate"]]
    if kind == "norm_fwd":
        yhat, mpost, spost = _normalised64(s["y"].double(), case["post"])
        h = s["scale_r"] * s["r"].double() + gate * _affine64(yhat, s["wpost"], s["bpost"])
        hhat, mpre, spre = _normalised64(h, case["pre"])
        return {"h": h, "v": _affine64(hhat, s["wpre"], s["bpre"]), "mpost": mpost, "spost": spost, "mpre": mpre,
                "spre": spre}
    hats = {}
    for side, x in (("pre", s["h"]), ("post", s["y"])):
        x = x.double()
        x = x if s["m" + side] is None else x - s["m" + side].double()
        hats[side] = x if s["s" + side] is None else x * s["s" + side].double()
    dv = s["dv"].double()
    dh = s["dh"].double() + _input_grad64(dv, s["wpre"], hats["pre"], s["spre"], case["pre"])
    dt = dh * gate
    dg = None
    if g is not None:
        slope = {"plain": 1.0, "sigmoid": p - p * p, "silu": p + g * (p - p * p)}[case["gate"]]
        dg = dh * slope * _affine64(hats["post"], s["wpost"], s["bpost"])
    return {"dr": s["scale_r"] * dh, "dy": _input_grad64(dt, s["wpost"], hats["post"], s["spost"], case["post"]),
            "dg": dg, "dwpost": torch.einsum("dn,dn->d", dt, hats["post"]),
            "dbpost": dt.sum(dim=1) if s["bpost"] is not None else None,
            "dwpre": torch.einsum("dn,dn->d", dv, hats["pre"]),
            "dbpre": dv.sum(dim=1) if s["bpre"] is not None else None}
