"""The example's gradients through its router against autograd in 64 bits, the experts' rows held
fixed, and as a part of the whole gradient.

Bars: route_backward is fp32 with sums of E terms (the softmax's and its gradient's) and of `tokens`
or E terms in its products, each within (terms + 8) * 2^-23 of the sum of magnitudes; the gradient of
the input is rounded to bf16 after the sum of both parts, 2^-8 of it, and the experts' part before."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("mx4_experts", os.path.join(ROOT, "examples", "mx4_experts.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def reference(layer, x, dweights):
    """(dx, d router, their sums of magnitudes) of <dweights, weights(x)> in 64 bits."""
    xd, r = x.double().requires_grad_(), layer.router.double().requires_grad_()
    p = torch.softmax(xd @ r, dim=1)
    ids = torch.softmax(x.float() @ layer.router, dim=1).topk(layer.topk, dim=1)[1]
    top = p.gather(1, ids)
    weights = top / top.sum(1, keepdim=True)
    dx, dr = torch.autograd.grad((weights * dweights.double()).sum(), (xd, r))
    with torch.no_grad():
        # |d top| <= 2 sum |d weights| / total, |d l| <= 2 p max |d top|
        size = 4 * dweights.double().abs().sum(1, keepdim=True) / top.sum(1, keepdim=True) * p
        return dx, dr, size @ r.abs().t(), xd.abs().t() @ size


@pytest.mark.parametrize("E,dim,hidden,topk,tokens", [(4, 160, 224, 2, 33), (8, 64, 96, 1, 70), (16, 128, 64, 4, 5), (4, 64, 64, 4, 20)])
def test_router(example, E, dim, hidden, topk, tokens):
    layer = example.Experts(E, dim, hidden, topk, seed=3)
    g = torch.Generator(device="cuda").manual_seed(7)
    x = torch.randn((tokens, dim), generator=g, device="cuda").bfloat16()
    dw = torch.randn((tokens, topk), generator=g, device="cuda")
    kept = layer.route(x)[2]
    dx, dr = layer.route_backward(dw, kept)
    want_x, want_r, size_x, size_r = reference(layer, x, dw)
    # (the logits, sums of dim terms, shift every probability by as much as themselves)
    logits = x.float().abs() @ layer.router.abs()
    off = (4 * float(logits.max()) * (dim + 8) + 8 * E + 32) * 2.0 ** -23
    assert ((dx - want_x).abs() <= off * size_x).all()
    assert ((dr - want_r).abs() <= (off + tokens * 2.0 ** -23) * size_r).all()


@pytest.mark.parametrize("E,dim,hidden,topk,tokens", [(4, 160, 224, 2, 33), (8, 64, 96, 3, 300)])
def test_the_whole_gradient_has_both_parts(example, E, dim, hidden, topk, tokens):
    layer = example.Experts(E, dim, hidden, topk, seed=4)
    g = torch.Generator(device="cuda").manual_seed(8)
    x = torch.randn((tokens, dim), generator=g, device="cuda").bfloat16()
    dy = torch.randn((tokens, dim), generator=g, device="cuda").bfloat16()
    layer.forward(x, keep=True)
    kept, seen, plain = layer.kept, [], layer.route_backward

    def spy(dweights, routing):
        out = plain(dweights, routing)
        seen.append((dweights, *out))
        return out

    layer.route_backward = spy
    dx, _, _, dr = layer.backward(dy)
    layer.route_backward = lambda dweights, routing: (torch.zeros_like(seen[0][1]), seen[0][2])
    experts, _, _, _ = layer.backward(dy)
    dweights, part, drouter = seen[0]
    assert torch.equal(dr, drouter) and torch.equal(dx, (experts.float() + part).bfloat16()) and part.abs().max() > 0
    # the weights' gradient that it starts from: <dy, the expert's row>
    ys, pos = kept[-1], kept[5].view(tokens, topk).long()
    terms = dy.double()[:, None] * ys.double()[pos]
    assert ((dweights - terms.sum(2)).abs() <= (dim + 1) * 2.0 ** -23 * terms.abs().sum(2)).all()


def test_training_moves_the_router(example):
    layer, losses = example.train(steps=3, experts=4, dim=128, hidden=256, tokens=500)
    fresh = example.Experts(4, 128, 256, 2)
    assert not torch.equal(layer.router, fresh.router) and all(x > 0 for x in losses)
