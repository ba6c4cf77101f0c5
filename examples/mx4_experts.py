"""A mixture-of-experts layer on the library's 4-bit and expert operators.

    python examples/mx4_experts.py          # a few training steps, then decode steps

The layer routes every token to topk of its experts, each a two-matrix network
y = W2 silu(W1 x), and sums the experts' outputs with the router's weights:

  forward    ids -> sfc_moe_sort; x, gathered in that order -> 4 bits; the experts' product;
             silu; 4 bits; the second product; sfc_moe_combine
  backward   sfc_moe_combine_grad; each product's two gradients, the output gradient
             brought to 4 bits along both ways in one read; the gather's gradient is
             sfc_moe_combine without weights; the router's part by its formulas in fp32

The experts' rows start at multiples of 32, so that no block of 32 rows, which share a
scale in the weight gradient, crosses experts.  Master weights are bf16 and go to 4 bits
once a step; a served layer keeps the 4-bit weights only.
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2601_16294_amd import sfcops as so  # noqa: E402

ALIGN = 32


class Experts:
    def __init__(self, experts, dim, hidden, topk, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.E, self.topk = experts, topk
        self.router = torch.randn(dim, experts, generator=g, device="cuda") * dim ** -0.5
        self.w1 = (torch.randn(experts, hidden, dim, generator=g, device="cuda") * dim ** -0.5).bfloat16()
        self.w2 = (torch.randn(experts, dim, hidden, generator=g, device="cuda") * hidden ** -0.5).bfloat16()
        self.quantise()

    def quantise(self):
        """The weights in 4 bits: along their rows for the products, transposed for their gradients."""
        self.q, self.qt = [], []
        for w in (self.w1, self.w2):
            E, N, K = w.shape
            q, qt = so.mx4_empty(N, K, lead=(E,)), so.mx4_empty(K, N, lead=(E,))
            for e in range(E):
                so.sfc_mx4_quant(w[e], q[0][e], q[1][e], qt[0][e], qt[1][e])
            self.q.append(q)
            self.qt.append(qt)

    def route(self, x):
        """(ids, weights, what route_backward needs): the topk experts of each token and their shares."""
        p = torch.softmax(x.float() @ self.router, dim=1)
        top, ids = p.topk(self.topk, dim=1)
        total = top.sum(1, keepdim=True)
        weights = top / total
        return ids.to(torch.int32), weights, (x, p, ids, weights, total)

    def route_backward(self, dweights, kept):
        """(dx, d router) from the gradient of the weights, the choice of experts being fixed.
        weights = top / total:  d top = (d weights - <d weights, weights>) / total, 0 for the others;
        p = softmax(l):         d l = p (d p - <d p, p>);  l = x router."""
        x, p, ids, weights, total = kept
        dtop = (dweights - (dweights * weights).sum(1, keepdim=True)) / total
        dp = torch.zeros_like(p).scatter_(1, ids, dtop)
        dl = p * (dp - (dp * p).sum(1, keepdim=True))
        return dl @ self.router.t(), x.float().t() @ dl

    def forward(self, x, keep=False):
        T, dim = x.shape
        ids, weights, routing = self.route(x)
        rows = so.sfc_moe_sort_rows(ids.numel(), self.E, ALIGN if keep else 1)
        new = lambda *shape: torch.empty(shape, dtype=torch.int32, device="cuda")
        offsets, order, pos = new(self.E + 1), new(rows), new(ids.numel())
        so.sfc_moe_sort(ids, offsets, order, pos, align=ALIGN if keep else 1)
        xq = so.mx4_empty(rows, dim)
        so.sfc_mx4_quant(x, *xq, order=order, topk=self.topk)
        h = torch.empty(rows, self.w1.shape[1], dtype=torch.bfloat16, device="cuda")
        so.sfc_moe_gemm_mx4_ex(*xq, *self.q[0], offsets, h)
        a = torch.nn.functional.silu(h)
        aq = so.mx4_empty(rows, a.shape[1])
        so.sfc_mx4_quant(a, *aq)
        ys = torch.empty(rows, dim, dtype=torch.bfloat16, device="cuda")
        so.sfc_moe_gemm_mx4_ex(*aq, *self.q[1], offsets, ys)
        y = torch.empty_like(x)
        so.sfc_moe_combine(ys, pos, y, weights=weights)
        if keep:
            self.kept = (x, weights, routing, offsets, order, pos, h, a, ys)
        return y

    def backward(self, dy):
        """(dx, dw1, dw2, d router) of the last forward(keep=True)."""
        x, weights, routing, offsets, order, pos, h, a, ys = self.kept
        rows, dim, hidden = ys.shape[0], x.shape[1], a.shape[1]
        dys, dweights = torch.empty_like(ys), torch.empty_like(weights)
        so.sfc_moe_combine_grad(dy, ys, order, pos, weights, dys, dweights)

        def product_grad(g, act, act_order, wt, n_in, n_out):
            # the output gradient in 4 bits along its rows (for d act) and its columns (for dW)
            gq, gt, at = so.mx4_empty(rows, n_out), so.mx4_empty(n_out, rows), so.mx4_empty(n_in, rows)
            so.sfc_mx4_quant(g, *gq, *gt)
            so.sfc_mx4_quant(act, None, None, *at, order=act_order, topk=self.topk)
            dact = torch.empty(rows, n_in, dtype=torch.bfloat16, device="cuda")
            dw = torch.empty(self.E, n_out, n_in, device="cuda")
            so.sfc_moe_gemm_mx4_ex(*gq, *wt, offsets, dact)
            so.sfc_moe_wgrad_mx4_ex(*gt, *at, offsets, dw)
            return dact, dw

        da, dw2 = product_grad(dys, a, None, self.qt[1], hidden, dim)
        s = torch.sigmoid(h.float())
        dh = (da.float() * s * (1 + h.float() * (1 - s))).bfloat16()
        dxs, dw1 = product_grad(dh, x, order, self.qt[0], dim, hidden)
        dx = torch.empty_like(x)
        so.sfc_moe_combine(dxs, pos, dx)
        dx_router, drouter = self.route_backward(dweights, routing)
        return (dx.float() + dx_router).to(dx.dtype), dw1, dw2, drouter

    def step(self, dw1, dw2, drouter, lr):
        self.w1 -= (lr * dw1).bfloat16()
        self.w2 -= (lr * dw2).bfloat16()
        self.router -= lr * drouter
        self.quantise()


def train(steps=20, experts=8, dim=512, hidden=1024, tokens=2000, topk=2, lr=40.0, seed=0):
    """Fits the layer to the outputs of a random linear map; the losses, step by step."""
    g = torch.Generator(device="cuda").manual_seed(seed + 1)
    layer = Experts(experts, dim, hidden, topk, seed)
    x = torch.randn(tokens, dim, generator=g, device="cuda").bfloat16()
    target = x.float() @ torch.randn(dim, dim, generator=g, device="cuda") * dim ** -0.5
    losses = []
    for _ in range(steps):
        y = layer.forward(x, keep=True)
        diff = y.float() - target
        losses.append(diff.square().mean())
        _, dw1, dw2, drouter = layer.backward((2 * diff / diff.numel()).bfloat16())
        layer.step(dw1, dw2, drouter, lr)
    return layer, [float(v) for v in torch.stack(losses)]


def main():
    torch.cuda.set_device(0)
    layer, losses = train()
    print("loss", " ".join(f"{v:.3f}" for v in losses))
    for tokens in (1, 16):
        x = torch.randn(tokens, layer.router.shape[0], device="cuda").bfloat16()
        for _ in range(10):
            layer.forward(x)
        start, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        start.record()
        for _ in range(100):
            layer.forward(x)
        end.record()
        torch.cuda.synchronize()
        print(f"{tokens} tokens: {start.elapsed_time(end) * 10:.0f} us a layer")


if __name__ == "__main__":
    main()
