"""hm_layer_few against a 64-bit reference and against the same layer out of the library's other calls."""
import numpy as np
import pytest
import torch

import around_reference as A
import layer_reference as R
from paper_2508_09591_amd import binding as B

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32
KIND = {BF16: "bf16", F32: "f32"}


class Layer:
    """Weights of experts first .. first + here - 1, in 8 bits and as the numbers they stand for."""

    def __init__(self, here, H, F, seed=0, first=0):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        r = lambda *shape: torch.randn(shape, generator=g, device="cuda")
        both = lambda w: B.hm_quantize_weights(w, *B.alloc_weights8(*w.shape))
        self.H, self.F, self.first, self.here = H, F, first, here
        self.w13, self.w2 = both(r(here, 2 * F, H) / H ** 0.5), both(r(here, H, F) / F ** 0.5)

    def numbers(self):
        n = lambda pair, C: R.weight_values(pair[0].float().cpu().numpy().astype(np.float64), pair[1].cpu().numpy().astype(np.int64))[:, :, :C]
        return n(self.w13, self.H), n(self.w2, self.F)

    def run(self, x, logits, router, out=None, bias=None, dtype=BF16, workspace=None, stream=None):
        T = x.shape[0]
        ids = torch.full((T, router.K), 99, dtype=torch.int32, device="cuda")
        weights = torch.full((T, router.K), float("nan"), device="cuda")
        out = torch.full((T, self.H), float("nan"), dtype=dtype, device="cuda") if out is None else out
        workspace = B.alloc_layer_few_workspace(T, router, self.H, self.F).fill_(0xAB) if workspace is None else workspace
        B.hm_layer_few(x, logits, router, *self.w13, *self.w2, ids, weights, out, workspace, bias, self.first, stream=stream)
        return ids, weights, out


def check(layer, x, ids, weights, out):
    want, off = A.layer_few(x.double().cpu().numpy(), ids.cpu().numpy(), weights.double().cpu().numpy(), *layer.numbers(), layer.first,
                            3 if out.dtype == F32 else 2)
    got = out.double().cpu().numpy()
    assert np.isfinite(got).all()
    assert (np.abs(got - want) <= A.HALF[KIND[out.dtype]] * (np.abs(want) + off) + off).all()
    scale = np.linalg.norm(want)
    if scale > 0:   # the bound is a worst case's: in the norm errors average out
        assert np.linalg.norm(got - want) <= (2.0 ** -8 if out.dtype == BF16 else 2e-6) * scale


def inputs(T, E, H, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return torch.randn((T, H), generator=g, device="cuda").to(BF16), torch.randn((T, E), generator=g, device="cuda")


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("T,E,K,H,F", [(1, 8, 2, 512, 128), (1, 1, 1, 1, 1), (1, 16, 8, 130, 70), (2, 4, 4, 7, 9), (3, 9, 3, 129, 127), (5, 60, 6, 1030, 257),
                                       (16, 8, 2, 256, 144), (17, 8, 2, 256, 144), (17, 3, 3, 200, 120), (33, 2, 1, 384, 100), (64, 4, 2, 260, 136),
                                       (64, 40, 16, 136, 72), (16, 70, 64, 128, 16), (40, 1, 1, 300, 300), (1, 300, 8, 2048, 768)])
def test_every_size(T, E, K, H, F, dtype):
    layer, router = Layer(E, H, F, seed=T), B.Router(E, K, "softmax")
    x, logits = inputs(T, E, H, T + 1)
    ids, weights, out = layer.run(x, logits, router, dtype=dtype)
    want_ids, want_weights = torch.empty_like(ids), torch.empty_like(weights)
    B.hm_route(logits, router, want_ids, want_weights)
    assert torch.equal(ids, want_ids) and torch.equal(weights, want_weights)
    check(layer, x, ids, weights, out)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("T,E,K,H,F", [(64, 64, 1, 264, 136), (50, 40, 4, 520, 72), (33, 24, 2, 264, 700), (20, 16, 1, 264, 640), (30, 32, 2, 136, 120),
                                       (30, 32, 2, 4100, 120)])
def test_all_tokens_choose_the_same_expert(T, E, K, H, F, dtype):
    """More than 16 slots of one expert, though on average there are few: its weights are read again, by the first product and by the second,
    which goes by experts, or by columns with two pieces of an expert (F = 640 to bf16) or several experts a wave (F = 120)."""
    layer, router = Layer(E, H, F, seed=T), B.Router(E, K, "softmax")
    assert T > 16 and T * K <= 10 * E   # so that one reading of the weights serves 16 slots
    x, logits = inputs(T, E, H, T + 2)
    logits[:, 3] = 9.0
    logits[::7, 3] = -9.0   # not of every token: slots are apart
    ids, weights, out = layer.run(x, logits, router, dtype=dtype)
    assert (ids == 3).sum() == T - (T + 6) // 7 > 16
    check(layer, x, ids, weights, out)
    again = layer.run(x, logits, router, dtype=dtype)[2]
    assert torch.equal(out, again)


@pytest.mark.parametrize("first,here", [(0, 8), (8, 24), (31, 1), (0, 32)])
def test_some_of_the_experts_are_here(first, here):
    """Groups, a bias, logits in bf16, rows that lie apart; slots of experts elsewhere add nothing, and the ranks' parts add up."""
    T, E, K, H, F = 21, 32, 4, 264, 136
    layer = Layer(here, H, F, seed=3, first=first)
    router = B.Router(E, K, "sigmoid", groups=4, top_groups=2, group_best=2, scale=2.5)
    x, logits = inputs(T, E, H, 5)
    bias = torch.linspace(-0.1, 0.1, E, device="cuda")
    wide = torch.full((T, H + 3), float("nan"), dtype=BF16, device="cuda")
    wide[:, 1:H + 1] = x
    wide_logits = torch.full((T, E + 5), float("nan"), dtype=BF16, device="cuda")
    wide_logits[:, :E] = logits.to(BF16)
    ids, weights, out = layer.run(wide[:, 1:H + 1], wide_logits[:, :E], router, bias=bias, dtype=F32)
    want_ids, want_weights = torch.empty_like(ids), torch.empty_like(weights)
    B.hm_route(logits.to(BF16), router, want_ids, want_weights, bias)
    assert torch.equal(ids, want_ids) and torch.equal(weights, want_weights)
    check(layer, x, ids, weights, out)


@pytest.mark.parametrize("E,groups,top_groups", [(96, 32, 5), (68, 17, 3), (40, 20, 6)])
def test_a_router_of_many_groups(E, groups, top_groups):
    """More groups than the lanes that choose inside the first product: the choice is hm_route's, for one token and for many."""
    K, H, F = 5, 264, 136
    layer = Layer(E, H, F, seed=E)
    for score, bias in (("softmax", None), ("sigmoid", torch.linspace(-0.1, 0.1, E, device="cuda"))):
        router = B.Router(E, K, score, groups=groups, top_groups=top_groups, group_best=2, scale=2.5)
        for T, dtype in ((1, F32), (4, BF16), (5, F32), (40, BF16)):
            x, logits = inputs(T, E, H, T + groups)
            ids, weights, out = layer.run(x, logits, router, bias=bias, dtype=dtype)
            want_ids, want_weights = torch.empty_like(ids), torch.empty_like(weights)
            B.hm_route(logits, router, want_ids, want_weights, bias)
            assert torch.equal(ids, want_ids) and torch.equal(weights, want_weights) and bool((ids >= 0).all())
            check(layer, x, ids, weights, out)


def test_tokens_without_experts_and_padded_ones():
    """-inf and NaN logits leave a token without slots: zeros, whatever its row holds; a NaN row stays its own."""
    T, E, K, H, F = 12, 6, 3, 200, 72
    layer, router = Layer(E, H, F), B.Router(E, K, "softmax")
    x, logits = inputs(T, E, H, 9)
    logits[3], logits[4] = float("-inf"), float("nan")
    logits[5, 2:] = float("-inf")
    clean = layer.run(x, logits, router)[2]
    x[3], x[4] = float("nan"), float("inf")
    ids, weights, out = layer.run(x, logits, router)
    assert torch.equal(out, clean) and not out[3:5].any() and (ids[3:5] == -1).all() and (ids[5] >= 0).sum() == 2
    x[3:5] = 0.0
    check(layer, x, ids, weights, out)
    x[7, 11] = float("nan")
    out = layer.run(x, logits, router)[2]
    others = [t for t in range(T) if t != 7]
    assert torch.isnan(out[7]).all() and torch.equal(out[others], clean[others])
    # nobody chooses anything
    logits[:] = float("-inf")
    assert not layer.run(x, logits, router)[2].any()


def test_an_expert_that_is_no_number_stays_its_tokens():
    T, E, K, H, F = 30, 4, 1, 256, 128
    layer, router = Layer(E, H, F), B.Router(E, K, "softmax")
    x, logits = inputs(T, E, H, 4)
    ids, _, clean = layer.run(x, logits, router)
    for pair in (layer.w13, layer.w2):
        scale = pair[1][2].clone()
        pair[1][2] = 255   # 2^128: as the conversion has it, no number that is finite
        out = layer.run(x, logits, router)[2]
        mine = (ids == 2).any(dim=1)
        assert mine.any() and torch.equal(out[~mine], clean[~mine]) and not torch.isfinite(out[mine]).all()
        pair[1][2] = scale


def test_no_tokens():
    layer, router = Layer(4, 128, 64), B.Router(4, 2)
    x, logits = inputs(0, 4, 128, 0)
    layer.run(x, logits, router)


def test_equal_tokens_get_equal_rows_wherever_they_stand():
    """A token's output does not depend on the others' number, place or choice."""
    E, K, H, F = 12, 4, 520, 264
    layer, router = Layer(E, H, F), B.Router(E, K)
    x, logits = inputs(64, E, H, 2)
    whole = layer.run(x, logits, router, dtype=F32)[2]
    for n in (1, 15, 16, 17, 32, 33):
        part = layer.run(x[:n], logits[:n], router, dtype=F32)[2]
        error = (part - whole[:n]).double().norm() / whole[:n].double().norm()
        assert error <= 2e-6   # the waves' shares of the sum go by the experts hit: another order of fp32 sums


def test_the_ways_through_a_graph_agree():
    """Eager, on another stream, through ctypes, captured and replayed with other inputs; two graphs with a workspace each."""
    E, K, H, F, T = 16, 4, 256, 128, 9
    layer, router = Layer(E, H, F), B.Router(E, K)
    x, logits = inputs(T, E, H, 2)
    workspace = B.alloc_layer_few_workspace(T, router, H, F)
    ids, weights, out = torch.empty((T, K), dtype=torch.int32, device="cuda"), torch.empty((T, K), device="cuda"), torch.empty((T, H), dtype=BF16, device="cuda")
    step = lambda stream=None: B.hm_layer_few(x, logits, router, *layer.w13, *layer.w2, ids, weights, out, workspace, stream=stream)
    step()
    want = out.clone()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        step()
    torch.cuda.synchronize()
    assert torch.equal(out, want)
    step(side)
    torch.cuda.synchronize()
    assert torch.equal(out, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for n in range(4):
        x2, logits2 = inputs(T, E, H, 20 + n)
        x.copy_(x2), logits.copy_(logits2)
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone()
        step()
        torch.cuda.synchronize()
        assert torch.equal(got, out)
        check(layer, x, ids, weights, out)
    # two calls at once, a workspace each
    others = [inputs(T, E, H, 50 + n) for n in range(2)]
    alone = [layer.run(*o, router)[2].clone() for o in others]
    streams, outs = [torch.cuda.Stream() for _ in range(2)], []
    torch.cuda.synchronize()
    for s, o in zip(streams, others):
        with torch.cuda.stream(s):
            outs.append(layer.run(*o, router)[2])
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(alone, outs))


def test_as_the_other_calls_have_it():
    """Route, plan, dispatch, products, activation and combine on the same weights; there x and the activation are in 8 bits."""
    E, K, H, F, T = 16, 4, 512, 256, 24
    layer, router = Layer(E, H, F), B.Router(E, K)
    x, logits = inputs(T, E, H, 2)
    ids, weights, out = layer.run(x, logits, router)
    plan = B.alloc_plan(T, K, E, 1, 1, B.HM_DEDUP_NONE, num_dest=E)
    B.hm_plan_mapped(ids, weights, torch.arange(E, dtype=torch.int32, device="cuda"), E, False, plan=plan)
    rows = torch.empty((T * K, H), dtype=BF16, device="cuda")
    B.hm_dispatch_pack(x, plan, rows)
    h = B.hm_expert_matmul(*B.hm_quantize_rows(rows, *B.alloc_rows8(T * K, H)), *layer.w13, plan.dest_offset, torch.empty((T * K, 2 * F), device="cuda"))
    _, *a8 = B.hm_gated(h, None, *B.alloc_rows8(T * K, F), offsets=plan.dest_offset)
    y = B.hm_expert_matmul(*a8, *layer.w2, plan.dest_offset, torch.empty((T * K, H), dtype=BF16, device="cuda"))
    other = B.hm_combine(y, None, plan, torch.empty((T, H), dtype=BF16, device="cuda"))
    # two roundings to 8 bits on the way, 2^-5.5 of a value each on average; silu amplifies less than twofold
    assert (other.double() - out.double()).norm() <= 3 * 2 ** -5.5 * out.double().norm()


def test_what_does_not_fit_is_refused():
    e = lambda *shape, dtype=BF16: torch.zeros(shape, dtype=dtype, device="cuda")
    layer, router = Layer(4, 128, 64), B.Router(8, 2)
    i32 = torch.int32
    ok = dict(x=e(3, 128), logits=e(3, 8), router=router, w13=layer.w13[0], w13_scale=layer.w13[1], w2=layer.w2[0], w2_scale=layer.w2[1],
              topk_ids=e(3, 2, dtype=i32), topk_weights=e(3, 2, dtype=F32), out=e(3, 128), bias=e(8, dtype=F32), first=4)
    call = lambda **k: B.hm_layer_few(**{**ok, **k})
    call()
    for bad in (dict(x=e(3, 256)), dict(x=e(128)), dict(logits=e(3, 7)), dict(logits=e(2, 8)), dict(w13=layer.w13[0][:, :127]), dict(w13_scale=layer.w13[1][:3]),
                dict(w2=layer.w2[0][:, :100]), dict(w2_scale=layer.w2[1][:, :0]), dict(topk_ids=e(3, 3, dtype=i32)), dict(topk_weights=e(2, 2, dtype=F32)),
                dict(out=e(3, 127)), dict(bias=e(7, dtype=F32))):
        with pytest.raises(ValueError):
            call(**bad)
    for bad in (dict(x=e(3, 128, dtype=F32)), dict(out=e(3, 128, dtype=torch.float16)), dict(topk_ids=e(3, 2, dtype=torch.int64)), dict(x=e(128, 3).t()),
                dict(w13=e(4, 128, 128))):
        with pytest.raises(TypeError):
            call(**bad)
    for bad in (dict(first=5), dict(first=-1), dict(workspace=e(64, dtype=torch.uint8)), dict(x=e(65, 128), logits=e(65, 8), topk_ids=e(65, 2, dtype=i32),
                                                                                             topk_weights=e(65, 2, dtype=F32), out=e(65, 128))):
        with pytest.raises(B.HierMoEError):
            call(**bad)
