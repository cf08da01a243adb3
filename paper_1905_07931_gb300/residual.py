"""A residual network of dense blocks under a compressed (CSR) classifier, trained with orthogonalised updates.

Each block is x <- x + W2 gelu(W1 x + b1) + b2 on bfloat16 activations (feature-major, d x n): two dense forward
products with bias, activation and residual in their epilogues, and backward the two products whose epilogues carry
gelu' and the residual's gradient, so that no elementwise pass runs between them. The classifier is a CSR layer in
float32 (Section 3.1) with softmax cross-entropy. The update direction of every weight matrix is the orthogonalised
momentum of its gradient: the blocks' matrices of one shape in one batched call, applied to float32 master weights;
the classifier's through the soft-threshold prox step (Section 2.2), which keeps it compressed. Biases take plain SGD.

    python -m paper_1905_07931_gb300.residual --steps 60
"""

from __future__ import annotations

import argparse
import json
import math

import torch

from . import csrtrain as C


class ResidualNet:
    """All buffers are allocated up front and every call is enqueued on the current stream (or ``stream``)."""

    def __init__(self, features: int, hidden: int, blocks: int, classes: int, batch: int, *, seed: int = 0,
                 density: float = 0.3, device="cuda", stream=None):
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
        self.ws = C.Workspace(classes, d, n, device=device, stream=stream)
        self.wsd = C.DenseWorkspace(max(d, h), max(d, h), n, device=device, stream=stream)
        self.ws1 = C.OrthogonalizeWorkspace(nb, h, d, device=device, stream=stream)
        self.ws2 = C.OrthogonalizeWorkspace(nb, d, h, device=device, stream=stream)
        self.wsc = C.OrthogonalizeWorkspace(1, classes, d, device=device, stream=stream)
        C.csr_from_dense(wc, self.wc[0], self.ws, stream)

    def forward(self):
        s = self.stream
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
        C.spmm_bwd_t(self.wc[self.cur], self.dlogits, self.dxf, self.ws, s)
        C.dense_act_bwd(self.dxf, None, "none", self.dx[self.L], stream=s)   # to bfloat16
        for i in range(self.L - 1, -1, -1):
            dy = self.dx[i + 1]
            C.dense_bwd_w(dy, self.a[i], self.g2[i], self.wsd, db=self.db2[i], stream=s)
            C.dense_bwd_x(self.w2h[i], dy, self.dz[i], self.wsd, z_below=self.z[i], act="gelu", stream=s)
            C.dense_bwd_w(self.dz[i], self.x[i], self.g1[i], self.wsd, db=self.db1[i], stream=s)
            C.dense_bwd_x(self.w1h[i], self.dz[i], self.dx[i], self.wsd, residual=dy, stream=s)

    def step(self, eta: float, lam: float, *, beta: float = 0.95, decay: float = 0.0):
        """One training step on ``x[0]`` / ``labels``; returns the device tensor whose element 0 is the mean loss."""
        s, d, h, nb = self.stream, self.d, self.h, self.L
        self.forward()
        C.softmax_xent(self.logits, self.labels, self.dlogits, self.loss, s)
        self.backward()
        scale = 0.2 * math.sqrt(max(d, h))
        C.orthogonalize(self.g1, self.o1, self.ws1, momentum=self.m1, beta=beta, scale=scale, stream=s)
        C.orthogonalize(self.g2, self.o2, self.ws2, momentum=self.m2, beta=beta, scale=scale, stream=s)
        C.dense_update(self.w1.view(nb * h, d), self.o1.view(nb * h, d), eta, decay, self.w1h.view(nb * h, d), stream=s)
        C.dense_update(self.w2.view(nb * d, h), self.o2.view(nb * d, h), eta, decay, self.w2h.view(nb * d, h), stream=s)
        C.dense_update(self.b1, self.db1, eta, stream=s)
        C.dense_update(self.b2, self.db2, eta, stream=s)
        # the classifier: the prox step along the orthogonalised direction, into the other CSR buffer
        C.orthogonalize(self.gc, self.oc, self.wsc, momentum=self.mc, beta=beta,
                        scale=0.2 * math.sqrt(max(self.classes, d)), stream=s)
        C.bias_grad_sgd(self.dlogits, self.bc, eta, None, s)
        C.prox_update_compact(self.wc[self.cur], self.oc, eta, lam, self.wc[1 - self.cur], self.ws, s)
        self.cur = 1 - self.cur
        return self.loss

    def status(self):
        """Device status flags of all workspaces, OR-ed (synchronises)."""
        flags = 0
        for ws in (self.ws, self.wsd, self.ws1, self.ws2, self.wsc):
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
    a = ap.parse_args(argv)
    net = ResidualNet(a.features, a.hidden, a.blocks, a.classes, a.batch, seed=a.seed)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(a.seed + 1)
    # classes around random centres
    centres = torch.randn(a.features, a.classes, generator=gen, device="cuda")
    for t in range(1, a.steps + 1):
        y = torch.randint(0, a.classes, (a.batch,), generator=gen, device="cuda")
        net.x[0].copy_(0.25 * centres[:, y] + torch.randn(a.features, a.batch, generator=gen, device="cuda"))
        net.labels.copy_(y)
        loss = net.step(a.eta, a.lam)
        if t == 1 or t % 10 == 0 or t == a.steps:
            w = net.wc[net.cur]
            print(json.dumps({"step": t, "loss": round(float(loss[0].item()), 5),
                              "classifier_density": round(w.nnz() / (w.rows * w.cols), 4), "status": net.status()}))


if __name__ == "__main__":
    main()
