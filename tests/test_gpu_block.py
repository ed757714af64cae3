"""The example layer with a norm in front, the activation's calls inside and the way for a few tokens, against 64 bits without
quantising, as they are used together."""
import pytest
import torch

from paper_2508_09591_amd import binding as B
from paper_2508_09591_amd import layer as L

pytestmark = pytest.mark.gpu

BF16 = torch.bfloat16


def inputs(T, H, seed, kept=None):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    r = lambda: torch.randn((T, H), generator=g, device="cuda")
    return r().to(BF16), r().to(BF16), None if kept is None else (2 * r()).to(kept), None if kept is None else r().to(kept)


def reference(layer, x, residual, gout, gtotal, ids):
    """Output, the sum that is kept, and the gradients by torch in 64 bits, with the choice that was made."""
    leaf = lambda t: t.detach().double().cpu().requires_grad_()
    x, gate, w13, w2, norm = (leaf(t) for t in (x, layer.gate, layer.w13, layer.w2, layer.norm))
    total = x if residual is None else x + residual.double().cpu()
    y = total * torch.rsqrt(total.square().mean(dim=1, keepdim=True) + layer.eps) * norm
    ids = ids.long().cpu()
    score = torch.softmax(y @ gate.t(), dim=1)
    w = torch.where(ids >= 0, score.gather(1, ids.clamp(min=0)), 0.0)
    w = w / w.sum(dim=1, keepdim=True)
    out = torch.zeros_like(x)
    for e in range(layer.E):
        t, k = (ids == e).nonzero(as_tuple=True)
        if len(t):
            h = y[t] @ w13[e].t()
            a = torch.nn.functional.silu(h[:, :layer.F]) * h[:, layer.F:]
            out = out.index_add(0, t, w[t, k][:, None] * (a @ w2[e].t()))
    loss = (out * gout.double().cpu()).sum()
    if gtotal is not None:
        loss = loss + (total * gtotal.double().cpu()).sum()
    loss.backward()
    return out.detach(), total.detach(), (x.grad, gate.grad, w13.grad, w2.grad, norm.grad)


def far(a, b):
    return float((a.double().cpu() - b).norm() / b.norm())


@pytest.mark.parametrize("T,E,K,H,F,kept", [(1, 8, 2, 512, 128, BF16), (200, 8, 2, 512, 320, torch.float32), (157, 16, 4, 1024, 200, BF16),
                                            (64, 12, 3, 512, 136, None)])
def test_norm_layer_and_gradients(T, E, K, H, F, kept):
    layer = L.make_layer(E, K, H, F, seed=T, norm=True)
    x, gout, residual, gtotal = inputs(T, H, T + 1, kept)
    out = layer.forward(x, residual)
    grads = layer.backward(gout, gtotal)
    want, total, want_grads = reference(layer, x, residual, gout, gtotal, layer.ids)
    if kept is not None:
        assert layer.total.dtype == kept and far(layer.total, total) <= 2 ** -8
    # e4m3 values are off by 2^-5.5 of themselves on average; two a product, up to three products in a row, with room (as the layer's
    # own test has it); the router's gradient is a small difference of large terms, so it and what it adds to the others has more
    assert far(out, want) <= 0.12
    for name, a, b in zip(("x", "w13", "w2", "norm"), (grads[0], *grads[2:]), (want_grads[0], *want_grads[2:])):
        assert torch.isfinite(a).all(), name
        assert far(a, b) <= 0.12, (name, far(a, b))
    assert torch.isfinite(grads[1]).all()


def size_of_the_router_gradient(layer, x, residual, gout, ids):
    """What the terms of the gate's gradient amount to.  A logit's gradient is a difference of dot products gout y, each a sum of H terms of
    either sign, and it is errors of the terms that add up, not of what is left of them."""
    total = (x if residual is None else x.double() + residual.double()).double().cpu()
    y = total * torch.rsqrt(total.square().mean(dim=1, keepdim=True) + layer.eps) * layer.norm.double().cpu()
    gate, w13, w2, gout, ids = (t.detach().cpu() for t in (layer.gate.double(), layer.w13.double(), layer.w2.double(), gout.double(), ids.long()))
    w = torch.softmax(y @ gate.t(), dim=1).gather(1, ids)
    w, length = w / w.sum(dim=1, keepdim=True), torch.zeros_like(w)
    for e in range(layer.E):
        t, k = (ids == e).nonzero(as_tuple=True)
        h = y[t] @ w13[e].t()
        length[t, k] = ((torch.nn.functional.silu(h[:, :layer.F]) * h[:, layer.F:]) @ w2[e].t()).norm(dim=1)
    size = gout.norm(dim=1, keepdim=True) * length / layer.H ** 0.5
    each = w * (size ** 2 + (w * size).square().sum(dim=1, keepdim=True)).sqrt()
    return (each.square().sum(dim=1) * y.square().sum(dim=1)).sum().sqrt()


@pytest.mark.parametrize("T,E,K,H,F,kept", [(200, 8, 2, 512, 320, torch.float32), (157, 16, 4, 1024, 200, BF16), (64, 12, 3, 512, 136, None)])
def test_the_layers_own_part_of_the_gradients(T, E, K, H, F, kept):
    """The gradient of x without what came past the layer, which is three to four times as large and would hide its errors, and the gate's."""
    layer = L.make_layer(E, K, H, F, seed=T, norm=True)
    x, gout, residual, gtotal = inputs(T, H, T + 1, kept)
    layer.forward(x, residual)
    grads = layer.backward(gout, gtotal)
    assert bool((layer.ids >= 0).all())
    want = reference(layer, x, residual, gout, None, layer.ids)[2]
    mine = grads[0].double() - (0 if gtotal is None else gtotal.double())
    # six values in 8 bits on the way, 2^-5.5 of each: 0.054, with room for the activation's share; that a sum four times as large is rounded
    # to bf16, 2^-9.8 of it on average, adds 0.005 of the part
    assert far(mine, want[0]) <= 0.12
    # the router's: y has four of the roundings, 0.044 of its terms, weights and x none; three times 0.05 as the layer's own test has it
    assert (grads[1].double().cpu() - want[1]).norm() <= 3 * 0.05 * size_of_the_router_gradient(layer, x, residual, gout, layer.ids)


@pytest.mark.parametrize("T,E,K,H,F,kept", [(1, 16, 4, 512, 256, BF16), (16, 8, 2, 1024, 320, torch.float32), (50, 32, 4, 512, 200, None)])
def test_few_tokens(T, E, K, H, F, kept):
    layer = L.make_layer(E, K, H, F, seed=T, norm=True)
    x, gout, residual, _ = inputs(T, H, T + 1, kept)
    whole = layer.forward(x, residual)
    ids = layer.ids
    few = layer.few(x, residual)
    want = reference(layer, x, residual, gout, None, ids)[0]
    # the weights alone are in 8 bits: 2^-5.5 a product on average, two of them, silu amplifying less than twofold
    assert far(few, want) <= 3 * 2 ** -5.5
    assert far(whole, want) <= 0.12
    assert far(few, want) < far(whole, want) or T == 1


def test_few_tokens_where_experts_are_gone():
    layer = L.make_layer(8, 4, 512, 64, norm=True)
    layer.gone = torch.arange(8, device="cuda") >= 3
    x, gout, residual, _ = inputs(20, 512, 3, BF16)
    layer.forward(x, residual)
    ids = layer.ids
    assert (ids >= 0).sum() == 60
    assert far(layer.few(x, residual), reference(layer, x, residual, gout, None, ids)[0]) <= 3 * 2 ** -5.5


def test_a_decoding_step_in_a_graph():
    """Norm, router's product, the layer: captured once, replayed for other tokens, with eager steps between."""
    layer = L.make_layer(16, 4, 512, 256, seed=9, norm=True)
    x, _, residual, _ = inputs(4, 512, 1, BF16)
    layer.few(x, residual)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = layer.few(x, residual)
        kept = layer.total
    for n in range(4):
        other, _, residual2, _ = inputs(4, 512, 10 + n, BF16)
        x.copy_(other), residual.copy_(residual2)
        graph.replay()
        torch.cuda.synchronize()
        eager = layer.few(x, residual)
        assert torch.equal(out, eager) and torch.equal(kept, layer.total)
        torch.cuda.synchronize()


def test_a_training_step_in_a_graph():
    """Forward and backward with the norm, captured while eager results of the same tensors live: the same gradients each time."""
    layer = L.make_layer(8, 2, 512, 128, seed=2, norm=True)
    x, gout, residual, gtotal = inputs(130, 512, 1, BF16)
    step = lambda: (layer.forward(x, residual), *layer.backward(gout, gtotal))
    want = [t.clone() for t in step()]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for _ in range(3):
        for t in got:
            t.fill_(7)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        again = step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(again, want))


def test_few_tokens_between_forward_and_backward():
    """A served batch changes nothing of what the way back reads."""
    layer = L.make_layer(8, 2, 512, 128, seed=3, norm=True)
    x, gout, residual, gtotal = inputs(20, 512, 4, BF16)
    layer.forward(x, residual)
    want = layer.backward(gout, gtotal)
    layer.forward(x, residual)
    x2, _, residual2, _ = inputs(20, 512, 9, BF16)
    layer.few(x2, residual2)
    assert torch.equal(layer.total, (x2.float() + residual2.float()).to(BF16))
    assert all(torch.equal(a, b) for a, b in zip(layer.backward(gout, gtotal), want))


def test_a_residual_needs_a_norm():
    layer = L.make_layer(8, 2, 512, 64)
    x, _, residual, _ = inputs(3, 512, 1, BF16)
    with pytest.raises(ValueError):
        layer.forward(x, residual)
    with pytest.raises(B.HierMoEError):
        layer.few(torch.zeros((65, 512), dtype=BF16, device="cuda"))


class _Recorder:
    """The native half with a note of each call: its name and whether it was taken."""
    def __init__(self, native):
        self.native, self.calls = native, []

    def __getattr__(self, name):
        def call(*args):
            rc = getattr(self.native, name)(*args)
            self.calls.append((name, rc is not None))
            return rc
        return call


def every_call(T, E, K, H, F, workspaces=True):
    """[(name, call(stream), its outputs)] of the calls around the products, on tensors of their own."""
    g = torch.Generator(device="cuda")
    g.manual_seed(T)
    r = lambda *shape, dtype=BF16: torch.randn(shape, generator=g, device="cuda").to(dtype)
    empty = lambda *shape, dtype=BF16: torch.empty(shape, dtype=dtype, device="cuda")
    x, past, weight, router = r(T, H), r(T, H), r(H, dtype=torch.float32), B.Router(E, K)
    total, y, y8, gx, gw = empty(T, H), empty(T, H), B.alloc_rows8(T, H), empty(T, H), empty(H, dtype=torch.float32)
    h, ga, a, offsets = r(T, 2 * F), r(T, F), empty(T, F), torch.tensor([0, T // 2, T], dtype=torch.int32, device="cuda")
    back8 = (*B.alloc_rows8(T, 2 * F), *(t.zero_() for t in (*B.alloc_columns8(T, 2, 2 * F), *B.alloc_columns8(T, 2, F))))
    w13 = B.hm_quantize_weights(r(E, 2 * F, H), *B.alloc_weights8(E, 2 * F, H))
    w2 = B.hm_quantize_weights(r(E, H, F), *B.alloc_weights8(E, H, F))
    logits, ids, w, out = r(T, E, dtype=torch.float32), empty(T, K, dtype=torch.int32), empty(T, K, dtype=torch.float32), empty(T, H)
    ws = (B.alloc_rms_norm_workspace(T, H), B.alloc_layer_few_workspace(T, router, H, F)) if workspaces else (None, None)
    return [("rms_norm", lambda s: B.hm_rms_norm(x, weight, 1e-6, y, *y8, past, total, stream=s), (total, y, *y8)),
            ("rms_norm_backward", lambda s: B.hm_rms_norm_backward(past, x, weight, 1e-6, gx, gw, None, ws[0], stream=s), (gx, gw)),
            ("gated", lambda s: B.hm_gated(h, a, None, None, offsets, stream=s), (a,)),
            ("gated_backward", lambda s: B.hm_gated_backward(h, ga, offsets, None, *back8, stream=s), back8),
            ("layer_few", lambda s: B.hm_layer_few(x, logits, router, *w13, *w2, ids, w, out, ws[1], stream=s), (ids, w, out))]


def test_ordinary_calls_are_the_native_halfs(monkeypatch):
    calls = every_call(20, 8, 2, 256, 128)
    rec = _Recorder(B._native)
    monkeypatch.setattr(B, "_native", rec)
    for _, call, _ in calls:
        call(None)
    torch.cuda.synchronize()
    assert rec.calls == [(name, True) for name, _, _ in calls]
    rec.calls.clear()
    for _, call, _ in calls:
        call(torch.cuda.current_stream())
    torch.cuda.synchronize()
    assert rec.calls == []   # a given stream is Python's


@pytest.mark.parametrize("name", ["rms_norm_backward", "layer_few"])
def test_scratch_of_a_call_belongs_to_its_stream(name):
    """A workspace that the call brings along is not given to the current stream while the call's own has yet to come to it."""
    rows = 40
    (_, call, outputs), = [c for c in every_call(rows, 8, 2, 256, 128, workspaces=False) if c[0] == name]
    need = B.alloc_rms_norm_workspace(rows, 256) if name == "rms_norm_backward" else B.alloc_layer_few_workspace(rows, B.Router(8, 2), 256, 128)
    need = need.numel()
    call(None)
    want = [t.clone() for t in outputs]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(50_000_000)
    call(side)
    mine = [torch.full((need,), 7, dtype=torch.uint8, device="cuda") for _ in range(4)]
    torch.cuda.current_stream().synchronize()
    torch.cuda.synchronize()
    assert all(bool((t == 7).all()) for t in mine)
    assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(outputs, want))


def far_apart(t, ld):
    """The same rows, ld elements apart, in memory of its own that is touched there alone."""
    wide = torch.empty((t.shape[0], ld), dtype=t.dtype, device="cuda")[:, :t.shape[1]]
    return wide.copy_(t)


def test_rows_whose_offsets_pass_32_bits():
    """Rows 2^29 elements apart, and for columns in 8 bits 1,100 rows 2^21 apart: the same bits as of rows that lie together."""
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    r = lambda *shape: torch.randn(shape, generator=g, device="cuda").to(BF16)
    T, H, F, ld = 5, 520, 260, 1 << 29
    x, past, gy, weight = r(T, H), r(T, H), r(T, H), r(H)
    empty = lambda *shape: torch.empty(shape, dtype=BF16, device="cuda")

    def norm(x, past, total):
        return B.hm_rms_norm(x, weight, 1e-6, empty(T, H), *B.alloc_rows8(T, H), past, total)
    want, total = norm(x, past, empty(T, H)), empty(T, ld)[:, :H]
    got = norm(far_apart(x, ld), far_apart(past, ld), total)
    assert all(torch.equal(a.contiguous().view(torch.uint8), b.view(torch.uint8)) for a, b in zip(got, want))
    gx, gw = empty(T, ld)[:, :H], torch.empty(H, device="cuda")
    B.hm_rms_norm_backward(far_apart(gy, ld), total, weight, 1e-6, gx, gw)
    gx2, gw2 = B.hm_rms_norm_backward(gy, want[3], weight, 1e-6, empty(T, H), torch.empty(H, device="cuda"))
    assert torch.equal(gx, gx2) and torch.equal(gw, gw2)
    del total, got, gx
    h, ga = r(T, 2 * F), r(T, F)
    assert torch.equal(B.hm_gated(far_apart(h, ld), empty(T, F))[0], B.hm_gated(h, empty(T, F))[0])
    assert torch.equal(B.hm_gated_backward(far_apart(h, ld), far_apart(ga, ld), gh=empty(T, 2 * F))[0], B.hm_gated_backward(h, ga, gh=empty(T, 2 * F))[0])
    E, K = 8, 2
    w13 = B.hm_quantize_weights(r(E, 2 * F, H), *B.alloc_weights8(E, 2 * F, H))
    w2 = B.hm_quantize_weights(r(E, H, F), *B.alloc_weights8(E, H, F))
    few = lambda x: B.hm_layer_few(x, logits, B.Router(E, K), *w13, *w2, torch.empty((T, K), dtype=torch.int32, device="cuda"),
                                   torch.empty((T, K), device="cuda"), empty(T, H))
    logits = r(T, E)
    assert torch.equal(few(far_apart(x, ld)), few(x))
    T, ld = 1100, 1 << 21
    h, ga, offsets = r(T, 2 * F), r(T, F), torch.tensor([0, 300, 1100], dtype=torch.int32, device="cuda")

    def columns(h, ga):
        outputs = [t.zero_() for t in (*B.alloc_columns8(T, 2, 2 * F), *B.alloc_columns8(T, 2, F))]
        return B.hm_gated_backward(h, ga, offsets, empty(T, 2 * F), None, None, *outputs)
    for a, b in zip(columns(far_apart(h, ld), far_apart(ga, ld)), columns(h, ga)):
        assert (a is None) == (b is None) and (a is None or torch.equal(a.view(torch.uint8), b.view(torch.uint8)))
