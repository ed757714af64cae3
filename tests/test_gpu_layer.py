"""The example layer: router, plan, dispatch, products, combine and the way back against 64 bits without quantising."""
import pytest
import torch

from paper_2508_09591_amd import binding as B
from paper_2508_09591_amd import layer as L

pytestmark = pytest.mark.gpu


def reference(layer, x, gout):
    """The layer in 64 bits with the choice that was made, its gradients by torch."""
    leaf = lambda t: t.detach().double().cpu().requires_grad_()
    x, gate, w13, w2, gout = leaf(x), leaf(layer.gate), leaf(layer.w13), leaf(layer.w2), gout.double().cpu()
    ids, router = layer.ids.long().cpu(), layer.router.c
    logits = x @ gate.t()
    score = torch.sigmoid(logits) if router.score == B.HM_SCORE_SIGMOID else torch.softmax(logits, dim=1)
    w = torch.where(ids >= 0, score.gather(1, ids.clamp(min=0)), 0.0)
    if router.renormalise:
        w = w / w.sum(dim=1, keepdim=True)
    u, w = w, w * router.scale
    out, length = torch.zeros_like(x), torch.zeros_like(w)
    for e in range(layer.E):
        t, k = (ids == e).nonzero(as_tuple=True)
        if len(t):
            h = x[t] @ w13[e].t()
            a = torch.nn.functional.silu(h[:, :layer.F]) * h[:, layer.F:]
            y = a @ w2[e].t()
            length[t, k] = y.detach().norm(dim=1)
            out = out.index_add(0, t, w[t, k][:, None] * y)
    out.backward(gout)
    # The router's gradient is a difference of dot products gout y, each a sum of H terms of either sign: what an error of
    # `share` of the values of y amounts to, by the size of the terms, as they cancel in the result.
    size = gout.norm(dim=1, keepdim=True) * length / gout.shape[1] ** 0.5
    each = router.scale * u.detach() * (size ** 2 + (u.detach() * size).square().sum(dim=1, keepdim=True)).sqrt()
    gate_error = (each.square().sum(dim=1) * x.detach().square().sum(dim=1)).sum().sqrt()
    return out.detach(), x.grad, gate.grad, w13.grad, w2.grad, gate_error


@pytest.mark.parametrize("T,E,K,H,F,score,how", [(1, 8, 2, 512, 64, "softmax", {}), (300, 8, 2, 512, 320, "softmax", {}),
                                                  (517, 64, 6, 512, 136, "sigmoid", dict(scale=2.5)),
                                                  (257, 16, 4, 1024, 256, "softmax", dict(renormalise=False)),
                                                  (129, 32, 4, 512, 200, "sigmoid", dict(groups=4, top_groups=2, group_best=2))])
def test_layer_and_its_gradients(T, E, K, H, F, score, how):
    layer = L.make_layer(E, K, H, F, score, seed=T, **how)
    g = torch.Generator(device="cuda")
    g.manual_seed(T + 1)
    x, gout = (torch.randn((T, H), generator=g, device="cuda").to(torch.bfloat16) for _ in range(2))
    out = layer.forward(x)
    grads = layer.backward(gout)
    want = reference(layer, x, gout)
    # An e4m3 value is off by at most 2^-4 and on average by 2^-5.5 of itself; two quantised operands a product, two products in a
    # row (three for the first weights): sqrt(2 * 3) * 2^-5.5 = 0.05, with room for activations that amplify.  The router's
    # gradient: three times 0.05 of what its terms amount to.
    for name, a, b in zip(("out", "x", "gate", "w13", "w2"), (out, *grads), want[:5]):
        a = a.double().cpu()
        assert torch.isfinite(a).all(), name
        bound = 3 * 0.05 * want[5] if name == "gate" else 0.12 * b.norm()
        assert (a - b).norm() <= bound, (name, float((a - b).norm() / b.norm()))


@pytest.mark.parametrize("score,how", [("softmax", {}), ("sigmoid", dict(scale=2.5)), ("sigmoid", dict(renormalise=False))])
def test_gradients_where_experts_are_gone(score, how):
    """Three of eight experts are left to four slots: every gradient is finite and right for those, and 0 for the others."""
    T, E, K, H, F, left = 90, 8, 4, 512, 64, 3
    layer = L.make_layer(E, K, H, F, score, seed=5, **how)
    layer.gone = torch.arange(E, device="cuda") >= left
    g = torch.Generator(device="cuda")
    g.manual_seed(6)
    x, gout = (torch.randn((T, H), generator=g, device="cuda").to(torch.bfloat16) for _ in range(2))
    out = layer.forward(x)
    grads = layer.backward(gout)
    assert (layer.ids >= 0).sum() == T * left and int(layer.ids.max()) < left
    want = reference(layer, x, gout)
    for name, a, b in zip(("out", "x", "gate", "w13", "w2"), (out, *grads), want[:5]):   # bounds as above
        a = a.double().cpu()
        assert torch.isfinite(a).all(), name
        bound = 3 * 0.05 * want[5] if name == "gate" else 0.12 * b.norm()
        assert (a - b).norm() <= bound, (name, float((a - b).norm() / b.norm()))
        assert name in ("out", "x") or not a[left:].any()


def test_dropped_slots_leave_rows_unused():
    """Experts of a rank that is gone: their logits are -inf, tokens that find too few are left with fewer slots."""
    layer = L.make_layer(8, 4, 512, 64)
    x = torch.randn((90, 512), device="cuda").to(torch.bfloat16)
    layer.gate = torch.where(torch.arange(8, device="cuda")[:, None] < 3, layer.gate, float("nan"))
    out = layer.forward(x)
    assert (layer.ids >= 0).sum() == 90 * 3 and int(layer.plan.dest_offset[8]) == 90 * 3
    assert torch.isfinite(out).all()
    for g in layer.backward(torch.ones_like(x))[2:]:
        assert torch.isfinite(g).all() and not g[3:].any()
