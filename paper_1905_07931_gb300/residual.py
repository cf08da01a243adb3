"""A residual network of dense blocks under a compressed (CSR) classifier, trained with orthogonalised updates.

Each block is x <- x + W2 gelu(W1 x + b1) + b2 on bfloat16 activations (feature-major, d x n): two dense forward
products with bias, activation and residual in their epilogues, and backward the two products whose epilogues carry
gelu' and the residual's gradient, so that no elementwise pass runs between them. The classifier is a CSR layer in
float32 (Section 3.1) with softmax cross-entropy. The update direction of every weight matrix is the orthogonalised
momentum of its gradient: the blocks' matrices of one shape in one batched call, applied to float32 master weights;
the classifier's through the soft-threshold prox step (Section 2.2), which keeps it compressed. Biases take plain SGD.

With ``norm`` the blocks are normed: v = pre(h), y = W2 gelu(W1 v + b1) + b2, h <- r_scale h + a(Wg v) post(y), on a
float32 stream h, with a norm before the classifier too. What lies between two blocks' products is one call each way
(block_norm_fwd, block_norm_bwd). With ``vocab`` the input is tokens, looked up in a trained table; with ``clip`` all
gradients are scaled to a global norm of at most that before any update.

    python -m paper_1905_07931_gb300.residual --steps 60
    python -m paper_1905_07931_gb300.residual --norm rms --gate silu --vocab 1000 --clip 1 --steps 60
"""

from __future__ import annotations

import argparse
import json
import math

import torch

from . import csrtrain as C


class ResidualNet:
    """All buffers are allocated up front and every call is enqueued on the current stream (or ``stream``).

    norm: None, "rms" or "layer", the kind of the norms before and after each block; gate (with norm): None, "none"
    (the product itself), "sigmoid" or "silu"; vocab: tokens in ``tokens`` instead of features in ``x[0]``; clip: the
    largest global gradient norm."""

    def __init__(self, features: int, hidden: int, blocks: int, classes: int, batch: int, *, seed: int = 0,
                 density: float = 0.3, device="cuda", stream=None, norm: str | None = None, gate: str | None = None,
                 r_scale: float = 1.0, vocab: int | None = None, clip: float | None = None):
        if gate is not None and norm is None:
            raise ValueError("a gate needs norm")
        self.d, self.h, self.L, self.classes, self.n = features, hidden, blocks, classes, batch
        self.stream = stream
        gen = torch.Generator(device=device)
        gen.manual_seed(seed)
        f32 = dict(dtype=torch.float32, device=device)
        b16 = dict(dtype=torch.bfloat16, device=device)
        d, h, n, nb = features, hidden, batch, blocks

        def normal(*shape, std):
            return torch.randn(*shape, generator=gen, **f32) * std

        # float32 master weights, stacked over the blocks, and their 16-bit copies
        self.w1, self.w2 = normal(nb, h, d, std=1 / math.sqrt(d)), normal(nb, d, h, std=0.5 / math.sqrt(h * nb))
        self.w1h, self.w2h = self.w1.to(torch.bfloat16), self.w2.to(torch.bfloat16)
        self.b1, self.b2 = torch.zeros(nb, h, **f32), torch.zeros(nb, d, **f32)
        self.g1, self.g2 = torch.zeros_like(self.w1), torch.zeros_like(self.w2)
        self.m1, self.m2 = torch.zeros_like(self.w1), torch.zeros_like(self.w2)
        self.o1, self.o2 = torch.zeros_like(self.w1), torch.zeros_like(self.w2)
        self.db1, self.db2 = torch.zeros_like(self.b1), torch.zeros_like(self.b2)
        # activations: x[i] enters block i, x[nb] leaves the last
        self.x = torch.zeros(nb + 1, d, n, **b16)
        self.z = torch.zeros(nb, h, n, **b16)
        self.a = torch.zeros(nb, h, n, **b16)
        self.dx = torch.zeros(nb + 1, d, n, **b16)
        self.dz = torch.zeros(nb, h, n, **b16)
        # classifier
        self.xf, self.dxf = torch.zeros(d, n, **f32), torch.zeros(d, n, **f32)
        self.logits, self.dlogits = torch.zeros(classes, n, **f32), torch.zeros(classes, n, **f32)
        self.labels = torch.zeros(n, dtype=torch.int32, device=device)
        self.loss = torch.zeros(n + 1, **f32)
        self.bc = torch.zeros(classes, **f32)
        self.gc, self.mc, self.oc = (torch.zeros(classes, d, **f32) for _ in range(3))
        wc = normal(classes, d, std=1 / math.sqrt(d))
        wc = wc * (torch.rand(classes, d, generator=gen, device=device) < density)
        self.wc = [C.CSR(classes, d, device=device), C.CSR(classes, d, device=device)]
        self.cur = 0
        self.norm, self.gate, self.r_scale, self.vocab, self.clip = norm, gate, r_scale, vocab, clip
        self.grads = [self.g1, self.g2, self.gc, self.db1, self.db2]
        self.extra_ws = []
        if norm is not None:
            # the stream between the blocks, and what each block (the classifier: the last) reads of it
            self.hs, self.v = torch.zeros(nb + 1, d, n, **f32), torch.zeros(nb + 1, d, n, **b16)
            self.y, self.dy = torch.zeros(nb, d, n, **b16), torch.zeros(nb, d, n, **b16)
            self.dv, self.dh = torch.zeros(nb + 1, d, n, **b16), torch.zeros(nb + 1, d, n, **f32)
            # weights and biases of the norms (rows: before block i or the classifier; after block i), gradients, statistics
            self.wn, self.dwn = torch.ones(2 * nb + 1, d, **f32), torch.zeros(2 * nb + 1, d, **f32)
            self.bn, self.dbn = torch.zeros(2 * nb + 1, d, **f32), torch.zeros(2 * nb + 1, d, **f32)
            self.mean, self.rstd = torch.zeros(2 * nb + 1, n, **f32), torch.zeros(2 * nb + 1, n, **f32)
            norms = [C.Norm(norm, self.wn[k], self.bn[k], mean=self.mean[k], rstd=self.rstd[k], dweight=self.dwn[k],
                            dbias=self.dbn[k]) for k in range(2 * nb + 1)]
            self.pre, self.post = norms[:nb + 1], norms[nb + 1:]
            self.wsn = C.BlockNormWorkspace(d, n, device=device, stream=stream)
            self.extra_ws.append(self.wsn)
            self.grads += [self.dwn, self.dbn]
        if gate is not None:
            self.wg = normal(nb, d, d, std=1 / math.sqrt(d))
            self.wgh = self.wg.to(torch.bfloat16)
            self.gg, self.mg, self.og = (torch.zeros_like(self.wg) for _ in range(3))
            self.z_gate, self.dz_gate = torch.zeros(nb, d, n, **b16), torch.zeros(nb, d, n, **b16)
            self.wsg = C.OrthogonalizeWorkspace(nb, d, d, device=device, stream=stream)
            self.extra_ws.append(self.wsg)
            self.grads.append(self.gg)
        if vocab is not None:
            self.table, self.dtable = normal(vocab, d, std=1 / math.sqrt(d)), torch.zeros(vocab, d, **f32)
            self.tokens = torch.zeros(n, dtype=torch.int32, device=device)
            self.wse = C.EmbedWorkspace(vocab, d, n, device=device, stream=stream)
            self.extra_ws.append(self.wse)
            self.grads.append(self.dtable)
        if clip is not None:
            self.dbc = torch.zeros(classes, **f32)   # else its update takes the sums as they are made
            self.grads.append(self.dbc)
            self.grad_norm = torch.zeros(2, **f32)
            self.wsk = C.GradWorkspace(device=device, stream=stream)
            self.extra_ws.append(self.wsk)
            self.grad_list = C.TensorList(self.grads)
        self.ws = C.Workspace(classes, d, n, device=device, stream=stream)
        self.wsd = C.DenseWorkspace(max(d, h), max(d, h), n, device=device, stream=stream)
        self.ws1 = C.OrthogonalizeWorkspace(nb, h, d, device=device, stream=stream)
        self.ws2 = C.OrthogonalizeWorkspace(nb, d, h, device=device, stream=stream)
        self.wsc = C.OrthogonalizeWorkspace(1, classes, d, device=device, stream=stream)
        C.csr_from_dense(wc, self.wc[0], self.ws, stream)

    def _norms_forward(self):
        s = self.stream
        if self.vocab is not None:
            C.embed_fwd(self.table, self.tokens, self.hs[0], self.wse, scale=math.sqrt(self.d), stream=s)
        else:
            C.dense_act_bwd(self.x[0], None, "none", self.hs[0], stream=s)   # to float32
        C.block_norm_fwd(None, self.hs[0], None, self.v[0], pre=self.pre[0], stream=s)
        for i in range(self.L):
            v, g = self.v[i], None
            C.dense_fwd(self.w1h[i], v, self.a[i], self.wsd, bias=self.b1[i], act="gelu", z=self.z[i], stream=s)
            C.dense_fwd(self.w2h[i], self.a[i], self.y[i], self.wsd, bias=self.b2[i], stream=s)
            if self.gate is not None:
                g = self.z_gate[i]
                C.dense_fwd(self.wgh[i], v, g, self.wsd, stream=s)
            C.block_norm_fwd(self.y[i], self.hs[i], self.hs[i + 1], self.v[i + 1], post=self.post[i], pre=self.pre[i + 1],
                             gate=g, gate_act=self.gate or "none", r_scale=self.r_scale, stream=s)
        return self.v[self.L]

    def _norms_backward(self):
        """From dv[L], the gradient of what the classifier reads, to dh[0], the stream's at the input."""
        s = self.stream
        for i in range(self.L - 1, -1, -1):
            v, gated = self.v[i], self.gate is not None
            C.block_norm_bwd(self.dv[i + 1], self.dh[i + 1] if i + 1 < self.L else None, self.hs[i + 1], self.y[i], self.dh[i],
                             self.dy[i], self.wsn, post=self.post[i], pre=self.pre[i + 1],
                             gate=self.z_gate[i] if gated else None, gate_act=self.gate or "none",
                             dgate=self.dz_gate[i] if gated else None, r_scale=self.r_scale, stream=s)
            C.dense_bwd_w(self.dy[i], self.a[i], self.g2[i], self.wsd, db=self.db2[i], stream=s)
            C.dense_bwd_x(self.w2h[i], self.dy[i], self.dz[i], self.wsd, z_below=self.z[i], act="gelu", stream=s)
            C.dense_bwd_w(self.dz[i], v, self.g1[i], self.wsd, db=self.db1[i], stream=s)
            C.dense_bwd_x(self.w1h[i], self.dz[i], self.dv[i], self.wsd, stream=s)
            if gated:
                C.dense_bwd_w(self.dz_gate[i], v, self.gg[i], self.wsd, stream=s)
                C.dense_bwd_x(self.wgh[i], self.dz_gate[i], self.dv[i], self.wsd, residual=self.dv[i], stream=s)
        dh = self.dh[0]
        C.block_norm_bwd(self.dv[0], dh if self.L else None, self.hs[0], None, dh, None, self.wsn, pre=self.pre[0], stream=s)
        return dh

    def forward(self):
        s = self.stream
        if self.norm is not None:
            C.dense_act_bwd(self._norms_forward(), None, "none", self.xf, stream=s)   # to float32
            C.spmm_fwd_bias_act(self.wc[self.cur], self.xf, self.bc, False, self.logits, self.ws, s)
            return self.logits
        if self.vocab is not None:
            C.embed_fwd(self.table, self.tokens, self.x[0], self.wse, scale=math.sqrt(self.d), stream=s)
        for i in range(self.L):
            C.dense_fwd(self.w1h[i], self.x[i], self.a[i], self.wsd, bias=self.b1[i], act="gelu", z=self.z[i], stream=s)
            C.dense_fwd(self.w2h[i], self.a[i], self.x[i + 1], self.wsd, bias=self.b2[i], residual=self.x[i], stream=s)
        C.dense_act_bwd(self.x[self.L], None, "none", self.xf, stream=s)   # to float32
        C.spmm_fwd_bias_act(self.wc[self.cur], self.xf, self.bc, False, self.logits, self.ws, s)
        return self.logits

    def backward(self):
        """Gradients of everything from ``dlogits`` (the classifier's bias is updated by the step)."""
        s = self.stream
        C.weight_grad_dense(self.dlogits, self.xf, self.gc, self.ws, C.CSRT_PREC_TF32, s)
        if self.clip is not None:
            C.bias_grad_sgd(self.dlogits, None, 0.0, self.dbc, s)
        C.spmm_bwd_t(self.wc[self.cur], self.dlogits, self.dxf, self.ws, s)
        if self.norm is not None:
            C.dense_act_bwd(self.dxf, None, "none", self.dv[self.L], stream=s)   # to bfloat16
            dx = self._norms_backward()
            if self.vocab is not None:
                C.embed_bwd(dx, self.tokens, self.dtable, self.wse, scale=math.sqrt(self.d), stream=s)
            return
        C.dense_act_bwd(self.dxf, None, "none", self.dx[self.L], stream=s)   # to bfloat16
        for i in range(self.L - 1, -1, -1):
            dy = self.dx[i + 1]
            C.dense_bwd_w(dy, self.a[i], self.g2[i], self.wsd, db=self.db2[i], stream=s)
            C.dense_bwd_x(self.w2h[i], dy, self.dz[i], self.wsd, z_below=self.z[i], act="gelu", stream=s)
            C.dense_bwd_w(self.dz[i], self.x[i], self.g1[i], self.wsd, db=self.db1[i], stream=s)
            C.dense_bwd_x(self.w1h[i], self.dz[i], self.dx[i], self.wsd, residual=dy, stream=s)
        if self.vocab is not None:
            C.embed_bwd(self.dx[0], self.tokens, self.dtable, self.wse, scale=math.sqrt(self.d), stream=s)

    def step(self, eta: float, lam: float, *, beta: float = 0.95, decay: float = 0.0):
        """One training step on ``x[0]`` (or ``tokens``) and ``labels``; returns the device tensor whose element 0 is the mean loss."""
        s, d, h, nb = self.stream, self.d, self.h, self.L
        self.forward()
        C.softmax_xent(self.logits, self.labels, self.dlogits, self.loss, s)
        self.backward()
        if self.clip is not None:
            C.grad_clip(self.grad_list, self.clip, self.grad_norm, self.wsk, stream=s)
        scale = 0.2 * math.sqrt(max(d, h))
        C.orthogonalize(self.g1, self.o1, self.ws1, momentum=self.m1, beta=beta, scale=scale, stream=s)
        C.orthogonalize(self.g2, self.o2, self.ws2, momentum=self.m2, beta=beta, scale=scale, stream=s)
        C.dense_update(self.w1.view(nb * h, d), self.o1.view(nb * h, d), eta, decay, self.w1h.view(nb * h, d), stream=s)
        C.dense_update(self.w2.view(nb * d, h), self.o2.view(nb * d, h), eta, decay, self.w2h.view(nb * d, h), stream=s)
        C.dense_update(self.b1, self.db1, eta, stream=s)
        C.dense_update(self.b2, self.db2, eta, stream=s)
        if self.norm is not None:
            C.dense_update(self.wn, self.dwn, eta, stream=s)
            C.dense_update(self.bn, self.dbn, eta, stream=s)
        if self.gate is not None:
            C.orthogonalize(self.gg, self.og, self.wsg, momentum=self.mg, beta=beta, scale=0.2 * math.sqrt(d), stream=s)
            C.dense_update(self.wg.view(nb * d, d), self.og.view(nb * d, d), eta, decay, self.wgh.view(nb * d, d), stream=s)
        if self.vocab is not None:
            C.dense_update(self.table, self.dtable, eta, stream=s)
        # the classifier: the prox step along the orthogonalised direction, into the other CSR buffer
        C.orthogonalize(self.gc, self.oc, self.wsc, momentum=self.mc, beta=beta,
                        scale=0.2 * math.sqrt(max(self.classes, d)), stream=s)
        if self.clip is not None:
            C.dense_update(self.bc.view(1, -1), self.dbc.view(1, -1), eta, stream=s)
        else:
            C.bias_grad_sgd(self.dlogits, self.bc, eta, None, s)
        C.prox_update_compact(self.wc[self.cur], self.oc, eta, lam, self.wc[1 - self.cur], self.ws, s)
        self.cur = 1 - self.cur
        return self.loss

    def status(self):
        """Device status flags of all workspaces, OR-ed (synchronises)."""
        flags = 0
        for ws in (self.ws, self.wsd, self.ws1, self.ws2, self.wsc, *self.extra_ws):
            flags |= ws.status(self.stream)[0]
        return flags


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--features", type=int, default=784)
    ap.add_argument("--hidden", type=int, default=1024)
    ap.add_argument("--blocks", type=int, default=3)
    ap.add_argument("--classes", type=int, default=10)
    ap.add_argument("--batch", type=int, default=256)
    ap.add_argument("--steps", type=int, default=60)
    ap.add_argument("--eta", type=float, default=0.003)
    ap.add_argument("--lam", type=float, default=0.1)
    ap.add_argument("--seed", type=int, default=0)
    ap.add_argument("--norm", choices=("rms", "layer"))
    ap.add_argument("--gate", choices=("none", "sigmoid", "silu"))
    ap.add_argument("--vocab", type=int, help="tokens as input, looked up in a table of so many rows")
    ap.add_argument("--clip", type=float, help="largest global norm of the gradients")
    a = ap.parse_args(argv)
    net = ResidualNet(a.features, a.hidden, a.blocks, a.classes, a.batch, seed=a.seed, norm=a.norm, gate=a.gate,
                      vocab=a.vocab, clip=a.clip)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(a.seed + 1)
    # classes around random centres
    centres = torch.randn(a.features, a.classes, generator=gen, device="cuda")
    for t in range(1, a.steps + 1):
        y = torch.randint(0, a.classes, (a.batch,), generator=gen, device="cuda")
        if a.vocab:   # a token's class is its remainder
            tokens = torch.randint(0, a.vocab, (a.batch,), generator=gen, device="cuda")
            net.tokens.copy_(tokens)
            y = tokens % a.classes
        else:
            net.x[0].copy_(0.25 * centres[:, y] + torch.randn(a.features, a.batch, generator=gen, device="cuda"))
        net.labels.copy_(y)
        loss = net.step(a.eta, a.lam)
        if t == 1 or t % 10 == 0 or t == a.steps:
            w = net.wc[net.cur]
            print(json.dumps({"step": t, "loss": round(float(loss[0].item()), 5),
                              "classifier_density": round(w.nnz() / (w.rows * w.cols), 4), "status": net.status(),
                              **({"grad_norm": round(float(net.grad_norm[0].item()), 5)} if a.clip else {})}))


if __name__ == "__main__":
    main()
