"""hm_route, hm_route_backward and hm_combine_weight_grad against 64-bit references."""
import numpy as np
import pytest
import torch

import layer_reference as R
from gpu_harness import dev
from paper_2508_09591_amd import binding as B

pytestmark = pytest.mark.gpu

# Relative error of a weight: exp and the division are good to a few units in the last place (2^-24), the exponent's
# argument loses |x - best| * 2^-24 (logits here span 20), and a sum of up to 4,096 terms, 64 in a lane, 70 * 2^-24.
RTOL = 1e-5


def grid(rng, T, E, step=0.125, span=6.0):
    """Logits that bf16 holds too and of which many are equal: what decides is either a tie or far apart."""
    return (np.round(rng.uniform(-span, span, (T, E)) / step) * step).astype(np.float32)


def run(x, router, bias=None, dtype=torch.float32, stride=0, stream=None):
    T, E = x.shape
    logits = torch.full((T, E + stride), float("nan"), dtype=dtype, device="cuda")[:, :E]
    logits.copy_(dev(x))
    ids = torch.full((T, router.K), 77, dtype=torch.int32, device="cuda")
    w = torch.full((T, router.K), float("nan"), device="cuda")
    if stream is not None:
        torch.cuda.synchronize()
    B.hm_route(logits, router, ids, w, None if bias is None else dev(bias), stream=stream)
    torch.cuda.synchronize()
    return logits, ids, w


def check(x, ids, w, bias, K, kind, **how):
    want, weights, gap = R.route(x, bias, K, kind, **how)
    assert gap > 1e-5, "the inputs do not decide beyond rounding"
    assert np.array_equal(ids.cpu().numpy(), want)
    got = w.cpu().numpy().astype(np.float64)
    assert np.all(np.abs(got - weights) <= RTOL * np.abs(weights) + 1e-37), np.abs(got - weights).max()


SHAPES = [(1, 256, 8), (3, 1, 1), (5, 2, 2), (130, 8, 2), (65, 16, 16), (64, 60, 6), (257, 64, 8), (33, 100, 10), (500, 128, 8),
          (129, 160, 5), (17, 255, 9), (4, 384, 33), (40, 512, 8), (6, 777, 12), (3, 1000, 1), (2, 4096, 64), (70, 257, 7)]


@pytest.mark.parametrize("kind,renormalise", [("softmax", True), ("softmax", False), ("sigmoid", True), ("sigmoid", False)])
@pytest.mark.parametrize("T,E,K", SHAPES)
def test_choice_and_weights(T, E, K, kind, renormalise):
    rng = np.random.default_rng(1000 * E + T)
    x = grid(rng, T, E)
    for dtype, stride in ((torch.float32, 0), (torch.bfloat16, 3), (torch.float32, 1), (torch.bfloat16, 8)):
        router = B.Router(E, K, kind, renormalise=renormalise, scale=2.5)
        _, ids, w = run(x, router, dtype=dtype, stride=stride)
        check(x, ids, w, None, K, kind, renormalise=renormalise, scale=2.5)


GROUPED = [(1, 256, 8, 8, 4, 2), (77, 256, 8, 8, 4, 2), (300, 64, 6, 8, 3, 1), (50, 60, 6, 5, 2, 2), (50, 60, 4, 15, 3, 2), (9, 512, 8, 16, 1, 2),
           (20, 24, 3, 24, 5, 1), (33, 128, 8, 2, 1, 2), (33, 128, 8, 4, 4, 2), (5, 1024, 10, 32, 7, 2), (12, 96, 8, 8, 4, 2), (12, 3000, 20, 100, 11, 2),
           (31, 288, 8, 8, 2, 2), (64, 512, 8, 4, 2, 1), (6, 160, 6, 8, 3, 2)]


@pytest.mark.parametrize("kind", ["softmax", "sigmoid"])
@pytest.mark.parametrize("T,E,K,groups,top,best", GROUPED)
def test_groups(T, E, K, groups, top, best, kind):
    rng = np.random.default_rng(E + groups)
    x = grid(rng, T, E, span=3.0)
    for dtype in (torch.float32, torch.bfloat16):
        _, ids, w = run(x, B.Router(E, K, kind, groups, top, best), dtype=dtype)
        check(x, ids, w, None, K, kind, groups=groups, top_groups=top, group_best=best)


@pytest.mark.parametrize("T,E,K,groups,top,best", GROUPED[:12] + [(200, 256, 8, 1, 1, 1), (3, 40, 40, 1, 1, 1), (100, 16, 4, 1, 1, 1)])
@pytest.mark.parametrize("kind", ["softmax", "sigmoid"])
def test_bias_chooses_and_does_not_weigh(T, E, K, groups, top, best, kind):
    """Scores of a few logits and biases on a grid of their own: sums are equal, or apart by far more than rounding."""
    rng = np.random.default_rng(7 * E + K)
    x = rng.choice(np.array([-1.5, 0.0, 0.75], dtype=np.float32), (T, E))
    bias = (rng.integers(-8, 9, E) * 0.0625).astype(np.float32)
    _, ids, w = run(x, B.Router(E, K, kind, groups, top, best, scale=0.5), bias)
    check(x, ids, w, bias, K, kind, groups=groups, top_groups=top, group_best=best, scale=0.5)


@pytest.mark.parametrize("kind", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renormalise", [True, False])
@pytest.mark.parametrize("groups", [1, 4])
@pytest.mark.parametrize("biased", [False, True])
def test_experts_that_cannot_be_chosen(kind, renormalise, groups, biased):
    """-inf and NaN are masks, +inf counts as the largest number, the lowest number is a number; rows with fewer experts than
    slots, with one and with none."""
    T, E, K = 24, 64, 6
    rng = np.random.default_rng(5)
    x = grid(rng, T, E, span=3.0)
    low = np.float32(np.finfo(np.float32).min)
    x[0] = -np.inf
    x[1] = np.nan
    x[2, 1:] = -np.inf
    x[3] = -np.inf
    x[3, [5, 40]] = 1.0
    x[4] = low
    x[5, ::2] = np.nan
    x[6, 7] = np.inf
    x[7, [7, 9]] = np.inf
    x[8] = np.where(rng.random(E) < 0.5, low, x[8])
    x[9, :32] = -np.inf
    x[10] = low
    x[10, 63] = 0.0
    x[11, ::3] = -np.inf
    x[12, 16:] = -np.inf
    x[13] = -200.0   # logistic scores of 0 in 32 bits
    bias = (rng.integers(-4, 5, E) * 0.5).astype(np.float32) if biased else None
    if biased:
        x[14:] = rng.choice(np.array([-1.5, 0.0, 0.75], dtype=np.float32), (T - 14, E))
        x[8, :] = np.where(x[8] == low, low, 0.5)
        x[[5, 9, 11, 12]] = np.where(np.isfinite(x[[5, 9, 11, 12]]), 0.25, x[[5, 9, 11, 12]])
        x[6, :] = np.where(np.isinf(x[6]), x[6], 0.25)
        x[7, :] = np.where(np.isinf(x[7]), x[7], 0.25)
    _, ids, w = run(x, B.Router(E, K, kind, groups, min(groups, 2), min(groups, 2), renormalise), bias)
    keep = np.ones(T, dtype=bool)
    if kind == "sigmoid":   # such scores may be 0: any weights between 0 and the exact ones
        keep[[4, 10, 13]] = False
        keep[8] = not np.any(x[8] == low)
    how = dict(groups=groups, top_groups=min(groups, 2), group_best=min(groups, 2), renormalise=renormalise)
    want, weights, gap = R.route(x, bias, K, kind, **how)
    got, got_w = ids.cpu().numpy(), w.cpu().numpy().astype(np.float64)
    assert np.array_equal(got[keep], want[keep])
    assert np.all(np.abs(got_w[keep] - weights[keep]) <= RTOL * weights[keep] + 1e-37)
    assert np.all(np.isfinite(got_w)) and np.all((got >= -1) & (got < E))
    assert np.all(got[:2] == -1) and np.all(got_w[:2] == 0)


def many(rng, T, E, bias, step):
    """Logits of which a token has many that are equal; with a bias three values and a grid for the bias, as above."""
    if bias:
        return rng.choice(np.array([-1.5, 0.0, 0.75], dtype=np.float32), (T, E)), (rng.integers(-8, 9, E) * 0.0625).astype(np.float32)
    return grid(rng, T, E, step), None


def check_some(x, ids, w, bias, K, kind, **how):
    """The first and the last tokens and some between against 64 bits."""
    T = len(x)
    some = np.unique(np.concatenate([np.arange(40), np.arange(T - 70, T), np.random.default_rng(T).integers(0, T, 200)]))
    check(x[some], ids[torch.from_numpy(some).cuda()], w[torch.from_numpy(some).cuda()], bias, K, kind, **how)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("kind,bias", [("softmax", False), ("sigmoid", False), ("sigmoid", True)])
@pytest.mark.parametrize("T,E,K", [(16384, 768, 8), (16385, 513, 3), (20001, 1000, 16)])
def test_more_experts_than_eight_lanes_hold(T, E, K, kind, bias, dtype):
    rng = np.random.default_rng(E)
    x, b = many(rng, T, E, bias, 0.125)
    _, ids, w = run(x, B.Router(E, K, kind), b, dtype=dtype)
    check_some(x, ids, w, b, K, kind)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("renormalise", [True, False])
@pytest.mark.parametrize("kind,bias", [("softmax", False), ("sigmoid", False), ("sigmoid", True)])
@pytest.mark.parametrize("T,E,K,groups,top,best", [(16384, 64, 8, 1, 1, 1), (16385, 60, 1, 1, 1, 1), (20001, 128, 3, 2, 1, 2), (16384, 256, 8, 8, 4, 2),
                                                  (17003, 96, 10, 8, 3, 2), (16390, 512, 16, 1, 1, 1), (16400, 40, 16, 4, 2, 1), (16384, 16, 2, 8, 2, 2),
                                                  (16387, 255, 9, 1, 1, 1), (16384, 5, 4, 1, 1, 1)])
def test_many_tokens(T, E, K, groups, top, best, kind, bias, renormalise, dtype):
    """What goes by eight lanes a token: lists of each length, two slots a lane, groups of one lane and of more, rows of any alignment."""
    rng = np.random.default_rng(T + E)
    x, b = many(rng, T, E, bias, 0.125)
    if groups > 1 and not bias:
        x = grid(rng, T, E, span=1.5 if E == 16 else 3.0)   # group scores apart by more than rounding
    elif groups == 1 and E > K:
        x[::5, E - 1] = -np.inf
    _, ids, w = run(x, B.Router(E, K, kind, groups, top, best, renormalise, 2.5), b, dtype=dtype, stride=(0, 1, 8)[E % 3])
    check_some(x, ids, w, b, K, kind, groups=groups, top_groups=top, group_best=best, renormalise=renormalise, scale=2.5)
    assert torch.all((ids >= 0) & (ids < E))
    again = run(x[-17:], B.Router(E, K, kind, groups, top, best, renormalise, 2.5), b, dtype=dtype)
    assert torch.equal(again[1], ids[-17:])   # 16 lanes a token choose alike


def test_no_tokens_and_another_stream():
    router = B.Router(16, 2)
    empty = torch.empty((0, 16), device="cuda")
    B.hm_route(empty, router, torch.empty((0, 2), dtype=torch.int32, device="cuda"), torch.empty((0, 2), device="cuda"))
    x = grid(np.random.default_rng(3), 40, 16)
    _, ids, w = run(x, router, stream=torch.cuda.Stream())
    check(x, ids, w, None, 2, "softmax")


def test_ids_go_straight_into_a_plan():
    """A slot that no expert is left for is one the router dropped: the plan skips it without an error."""
    T, E, K = 100, 16, 4
    x = grid(np.random.default_rng(9), T, E)
    x[::7, 3:] = -np.inf
    _, ids, w = run(x, B.Router(E, K))
    plan = B.hm_plan(ids, w, dev((np.arange(E) // 4).astype(np.int32)), 2, 2, B.HM_DEDUP_NONE)
    status, rows = B.hm_plan_status(plan)
    assert status == 0 and rows == int((ids >= 0).sum()) < T * K


# ---- the way back ---------------------------------------------------------------------------------------------------
def back(x, ids, g, router, dtype=torch.float32, stride=0):
    T, E = x.shape
    wide = lambda: torch.full((T, E + stride), float("nan"), dtype=dtype, device="cuda")
    logits, grad = wide()[:, :E], wide()
    logits.copy_(dev(x))
    B.hm_route_backward(logits, router, dev(ids.astype(np.int32)), dev(g), grad[:, :E])
    torch.cuda.synchronize()
    if stride:
        assert torch.isnan(grad[:, E:]).all()
    return grad[:, :E].float().cpu().numpy().astype(np.float64)


@pytest.mark.parametrize("kind,renormalise", [("softmax", True), ("softmax", False), ("sigmoid", True), ("sigmoid", False)])
@pytest.mark.parametrize("T,E,K", SHAPES + [(1, 8, 8), (2, 3, 3)])
def test_gradient_of_the_logits(T, E, K, kind, renormalise):
    """Against the formula, and against differences of the 64-bit forward pass."""
    rng = np.random.default_rng(E * K + T)
    x = grid(rng, T, E, span=4.0)
    ids = np.argsort(-x, axis=1, kind="stable")[:, :K]
    ids = np.take_along_axis(ids, rng.permuted(np.tile(np.arange(K), (T, 1)), axis=1), axis=1)
    if K > 1:
        ids[T // 2, K // 2] = -1
    g = rng.standard_normal((T, K)).astype(np.float32)
    router = B.Router(E, K, kind, renormalise=renormalise, scale=1.5)
    want, size = R.route_backward(x, ids, g, kind, renormalise, 1.5)
    got = back(x, ids, g, router)
    assert np.all(np.abs(got - want) <= RTOL * size + 1e-36), np.abs(got - want).max()
    half = back(x, ids, g, router, torch.bfloat16, 5)
    assert np.all(np.abs(half - want) <= (RTOL + 2.0 ** -8) * size + 1e-36)
    if E <= 128:   # differences: sum of g w around x, one logit at a time, for a few tokens
        for t in {0, T // 2, T - 1}:
            X, I = np.repeat(x[t:t + 1].astype(np.float64), E, axis=0), np.repeat(ids[t:t + 1], E, axis=0)
            f = lambda d: (R.weights_of(X + d * np.eye(E), I, kind, renormalise, 1.5) * g[t]).sum(axis=1)
            slope = (f(1e-5) - f(-1e-5)) / 2e-5
            # the difference's own error: h^2 / 6 of a third derivative, and 1e-16 / h of cancellation
            assert np.all(np.abs(got[t] - slope) <= RTOL * size[t] + 1e-9 * (1 + np.abs(g[t]).sum())), t


def test_gradient_where_experts_are_masked_or_ids_are_not_experts():
    T, E, K = 8, 32, 4
    rng = np.random.default_rng(2)
    x = grid(rng, T, E)
    x[1, 5:] = -np.inf
    x[2] = -np.inf
    x[3, :30] = np.nan
    x[4] = np.finfo(np.float32).min
    ids = np.argsort(-np.where(np.isnan(x), -np.inf, x), axis=1, kind="stable")[:, :K]
    ids[5, 2], ids[6, 1] = E + 3, -9
    g = rng.standard_normal((T, K)).astype(np.float32)
    for kind in ("softmax", "sigmoid"):
        for renormalise in (True, False):
            want, size = R.route_backward(x, ids, g, kind, renormalise, 1.0)
            got = back(x, ids, g, B.Router(E, K, kind, renormalise=renormalise))
            keep = np.arange(T) != (4 if kind == "sigmoid" else -1)   # scores of 0 in 32 bits
            assert np.all(np.abs(got - want)[keep] <= RTOL * size[keep] + 1e-36), (kind, renormalise)
            assert np.all(np.isfinite(got)) and np.all(got[2] == 0)


@pytest.mark.parametrize("level", [B.HM_DEDUP_NONE, B.HM_DEDUP_GPU, B.HM_DEDUP_NODE])
@pytest.mark.parametrize("T,K,H", [(1, 1, 1), (1, 8, 7168), (5, 3, 7), (70, 8, 512), (33, 6, 1030), (129, 9, 2049), (3, 64, 100), (260, 2, 64), (40, 10, 4097)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_gradient_of_the_weights(T, K, H, level, dtype):
    E, nodes, ranks = 64, 2, 4
    rng = np.random.default_rng(T + K + H)
    ids = np.argsort(rng.random((T, E)), axis=1)[:, :K].astype(np.int32)
    ids[rng.random((T, K)) < 0.1] = -1
    w = np.full((T, K), 0.5, dtype=np.float32)
    plan = B.hm_plan(dev(ids), dev(w), dev((np.arange(E) // 8).astype(np.int32)), nodes, ranks, level)
    status, rows = B.hm_plan_status(plan)
    assert status == 0
    off = 1 if H % 2 else 0   # rows off a vector's alignment
    flat = lambda n: torch.from_numpy(rng.standard_normal(n * H + off, dtype=np.float32)).cuda().to(dtype)[off:].view(n, H)
    gout, y = flat(T), flat(max(rows, 1))[:rows]
    grad = torch.full((T, K), float("nan"), device="cuda")
    B.hm_combine_weight_grad(gout, y, plan, grad)
    slot = plan.slot_row[:T * K].cpu().numpy().reshape(T, K)
    a, b = gout.double().cpu().numpy(), y.double().cpu().numpy()
    b = np.concatenate([b, np.zeros((1, H))])
    rows_of = b[np.where(slot >= 0, slot, rows)]
    want, size = (a[:, None] * rows_of).sum(axis=2), (np.abs(a)[:, None] * np.abs(rows_of)).sum(axis=2)
    # products of bf16 are exact, each of the lane's H / 64 additions and of the six after them rounds once
    bound = (H / 64 + 24) * 2.0 ** -24 * size
    assert np.all(np.abs(grad.cpu().numpy() - want) <= bound)
    assert B.hm_plan_status(plan)[0] == 0
    # rows that the buffer does not have count as zeros and are reported
    if rows > 1 and H > 1:
        B.hm_combine_weight_grad(gout, y[:rows - 1], plan, grad)
        want[slot == rows - 1], bound[slot == rows - 1] = 0, 0
        assert np.all(np.abs(grad.cpu().numpy() - want) <= bound)
        assert B.hm_plan_status(plan)[0] == B.HM_ERR_CAPACITY


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T,K,H", [(4097, 8, 512), (4101, 6, 1030), (4100, 9, 2049), (4099, 3, 4097), (4097, 8, 4608), (4097, 2, 520)])
def test_gradient_of_many_tokens_weights(T, K, H, dtype):
    """A wave to a token: rows of several steps, with a rest and without, slots in one piece and in several."""
    E, nodes, ranks = 64, 2, 4
    rng = np.random.default_rng(T + K + H)
    ids = np.argsort(rng.random((T, E)), axis=1)[:, :K].astype(np.int32)
    ids[rng.random((T, K)) < 0.1] = -1
    plan = B.hm_plan(dev(ids), dev(np.full((T, K), 0.5, dtype=np.float32)), dev((np.arange(E) // 8).astype(np.int32)), nodes, ranks, B.HM_DEDUP_NONE)
    status, rows = B.hm_plan_status(plan)
    assert status == 0
    g = torch.Generator(device="cuda")
    g.manual_seed(H)
    off = 1 if H % 2 else 0   # rows off a vector's alignment
    flat = lambda n: torch.randn(n * H + off, generator=g, device="cuda").to(dtype)[off:].view(n, H)
    gout, y, grad = flat(T), flat(rows), torch.full((T, K), float("nan"), device="cuda")
    B.hm_combine_weight_grad(gout, y, plan, grad)
    slot = plan.slot_row[:T * K].view(T, K).long()
    for some in torch.arange(T, device="cuda").split(512):
        row = slot[some]
        a, b = gout[some].double()[:, None], torch.where((row >= 0)[:, :, None], y[row.clamp(min=0)].double(), 0.0)
        want, size = (a * b).sum(dim=2), (a.abs() * b.abs()).sum(dim=2)
        # as in test_gradient_of_the_weights: H / 64 additions in a lane and six after them, each rounds once
        assert ((grad[some].double() - want).abs() <= (H / 64 + 24) * 2.0 ** -24 * size).all()
    assert B.hm_plan_status(plan)[0] == 0


@pytest.mark.parametrize("score,renormalise", [("softmax", False), ("softmax", True), ("sigmoid", True)])
def test_gradient_of_the_logits_of_many_tokens(score, renormalise):
    T, E, K = 20011, 60, 6
    rng = np.random.default_rng(6)
    x = grid(rng, T, E, span=4.0)
    ids = np.argsort(-x, axis=1, kind="stable")[:, :K]
    g = rng.standard_normal((T, K)).astype(np.float32)
    got = back(x, ids, g, B.Router(E, K, score, renormalise=renormalise, scale=1.5))
    want, size = R.route_backward(x, ids, g, score, renormalise, 1.5)
    assert np.all(np.abs(got - want) <= RTOL * size + 1e-36)


def test_the_weights_gradient_is_the_combines_derivative():
    """sum of gout * combine(w) is linear in w: its difference is the gradient."""
    T, E, K, H = 20, 16, 4, 96
    rng = np.random.default_rng(0)
    ids = np.argsort(rng.random((T, E)), axis=1)[:, :K].astype(np.int32)
    w, v = rng.random((T, K), dtype=np.float32), rng.random((T, K), dtype=np.float32)
    e2r = dev((np.arange(E) // 4).astype(np.int32))
    plan = B.hm_plan(dev(ids), dev(w), e2r, 2, 2, B.HM_DEDUP_NODE)
    _, rows = B.hm_plan_status(plan)
    y, gout = torch.randn((rows, H), device="cuda"), torch.randn((T, H), device="cuda")
    grad = torch.empty((T, K), device="cuda")
    B.hm_combine_weight_grad(gout, y, plan, grad)
    out = [B.hm_combine_f32(y, dev(u), plan, torch.empty((T, H), device="cuda")).double() for u in (w, v)]
    change = (gout.double() * (out[1] - out[0])).sum(dim=1).cpu().numpy()
    along = (grad.double().cpu().numpy() * (v.astype(np.float64) - w)).sum(axis=1)
    size = (gout.double().abs() * (out[0].abs() + out[1].abs())).sum(dim=1).cpu().numpy() + np.abs(grad.double().cpu().numpy()).sum(axis=1)
    assert np.all(np.abs(change - along) <= 64 * 2.0 ** -24 * size)


def test_replayed_in_a_graph():
    T, E, K = 300, 128, 8
    rng = np.random.default_rng(4)
    router = B.Router(E, K, "sigmoid", 8, 4, 2)
    logits, ids, w = torch.empty((T, E), device="cuda"), torch.empty((T, K), dtype=torch.int32, device="cuda"), torch.empty((T, K), device="cuda")
    g, grad = torch.randn((T, K), device="cuda"), torch.empty((T, E), device="cuda")
    calls = lambda: (B.hm_route(logits, router, ids, w), B.hm_route_backward(logits, router, ids, g, grad))
    logits.copy_(dev(grid(rng, T, E)))
    calls()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls()
    for _ in range(3):
        logits.copy_(dev(grid(rng, T, E)))
        calls()
        want = [t.clone() for t in (ids, w, grad)]
        for t in (ids, w, grad):
            t.fill_(7)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, (ids, w, grad)))
