"""hm_gated and its way back against 64-bit references, in values and both layouts of 8 bits."""
import numpy as np
import pytest
import torch

import around_reference as A
import layer_reference as R
from paper_2508_09591_amd import binding as B

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32
KIND = {BF16: "bf16", F32: "f32"}


def drawn(seed, rows, C, dtype, sigma=1.0):
    g = torch.Generator()
    g.manual_seed(seed)
    return (torch.randn((rows, C), generator=g) * torch.exp(torch.randn((rows, 1), generator=g)) * sigma).to(dtype)


def spaced(t, extra):
    rows, C = t.shape
    return torch.full((rows * (C + extra) + extra,), float("nan"), dtype=t.dtype, device="cuda")[extra:].view(rows, C + extra)[:, :C].copy_(t)


def f64(t):
    return t.double().cpu().numpy()


def poisoned(pair):
    for t in pair:
        t.view(torch.uint8).fill_(0xAB)
    return pair


def numbers8(pair):
    return pair[0].float().cpu().numpy().astype(np.float64), pair[1].cpu().numpy().astype(np.int64)


def is_poison(t):
    return bool((t.view(torch.uint8) == 0xAB).all())


SIZES = [(1, 1), (1, 2048), (3, 5), (2, 7), (7, 64), (5, 127), (65, 128), (9, 129), (33, 257), (4, 515), (130, 384), (3, 2056), (1, 4096)]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows,F", SIZES + [(20000, 520)])
def test_gated(rows, F, dtype):
    h = drawn(rows + F, rows, 2 * F, dtype, 2.0)
    want, off = A.gated(f64(h))
    for extra, atype in ((0, BF16), (3, F32)):
        a, pair = torch.full((rows, F), float("nan"), dtype=atype, device="cuda"), poisoned(B.alloc_rows8(rows, F))
        g = spaced(h, extra)
        B.hm_gated(g, a, *pair)
        assert (np.abs(f64(a) - want) <= A.HALF[KIND[atype]] * (np.abs(want) + off) + off).all()
        q, codes = numbers8(pair)
        A.check_rows8(q, codes, want, off)
        if atype == F32:
            want8, want_codes = R.rows8(f64(a))
            assert np.array_equal(q, want8) and np.array_equal(codes, want_codes)
        alone, only = torch.empty_like(a), B.alloc_rows8(rows, F)
        B.hm_gated(g, alone)
        B.hm_gated(g, None, *only)
        assert torch.equal(alone, a) and all(torch.equal(x.view(torch.uint8), y.view(torch.uint8)) for x, y in zip(only, pair))


def test_the_activation_where_it_saturates():
    gate = torch.tensor([0.0, -0.0, 1e-30, 20.0, 90.0, 3e38, -20.0, -87.0, -89.0, -104.0, -1000.0, -3e38, float("nan")])
    up = torch.tensor([3.0, -2.0, 1.0, 5.0, 1e-30, 0.5, 7.0, 1e20, 1e30, 1e38, 1e38, 2.0, 1.0])
    h = torch.cat([gate, up])[None].cuda()
    a = torch.empty((1, 13), device="cuda")
    B.hm_gated(h, a)
    want, off = A.gated(f64(h[:, :]))
    assert torch.isnan(a[0, 12])
    assert (np.abs(f64(a)[:, :12] - want[:, :12]) <= A.U * np.abs(want[:, :12]) + off[:, :12]).all()
    gh = torch.empty((1, 26), device="cuda")
    ga = torch.full((1, 13), 0.5, device="cuda")
    B.hm_gated_backward(h, ga, gh=gh)
    want, off = A.gated_backward(f64(h), f64(ga))
    fine = np.arange(26) % 13 < 12
    assert (np.abs(f64(gh) - want) <= A.U * np.abs(want) + off)[:, fine].all() and torch.isnan(gh[0, [12, 25]]).all()


# rows per segment: empty ones, one row, whole blocks, ends inside a block, none at all
COUNTS = [[5], [0, 1, 0], [128, 256, 1, 0, 127], [130, 3, 0, 259, 64], [0, 0, 0], [1] * 70, [0] * 100 + [200] + [0] * 30 + [77]]


@pytest.mark.parametrize("dtype,gtype", [(BF16, BF16), (F32, F32), (BF16, F32)])
@pytest.mark.parametrize("F", [1, 5, 64, 127, 128, 130, 256, 640, 1001])
@pytest.mark.parametrize("counts", range(len(COUNTS)))
def test_gated_backward(counts, F, dtype, gtype):
    """Every output of every row of a segment, and nothing of the rows before and behind them."""
    counts, before, behind = COUNTS[counts], 3 if F % 2 else 0, 4
    offsets = np.concatenate([[before], before + np.cumsum(counts)]).astype(np.int32)
    rows, S = int(offsets[-1]) + behind, len(counts)
    h, ga = drawn(rows + F, rows, 2 * F, dtype, 2.0), drawn(F, rows, F, dtype, 0.03)
    off_d = torch.from_numpy(offsets).cuda()
    gh = torch.full((rows, 2 * F), 7.0, dtype=gtype, device="cuda")
    rows8 = poisoned(B.alloc_rows8(rows, 2 * F))
    columns8, a8 = poisoned(B.alloc_columns8(rows, S, 2 * F)), poisoned(B.alloc_columns8(rows, S, F))
    extra = 3 if F % 2 else 0
    g_h, g_ga = spaced(h, 2 * extra), spaced(ga, extra)
    B.hm_gated_backward(g_h, g_ga, off_d, gh, *rows8, *columns8, *a8)
    in_segment = slice(before, int(offsets[-1]))
    want, off = A.gated_backward(f64(h), f64(ga))
    assert (np.abs(f64(gh) - want) <= A.HALF[KIND[gtype]] * (np.abs(want) + off) + off)[in_segment].all()
    for outside in (slice(0, before), slice(int(offsets[-1]), None)):
        assert bool((gh[outside] == 7.0).all()) and is_poison(rows8[0][outside]) and is_poison(rows8[1][outside])
    q, codes = numbers8(rows8)
    A.check_rows8(q[in_segment], codes[in_segment], want[in_segment], off[in_segment])
    # in fp32 the values are those that were rounded to 8 bits
    full = torch.zeros((rows, 2 * F), device="cuda")
    B.hm_gated_backward(g_h, g_ga, off_d, gh=full)
    want8, want_codes = R.rows8(f64(full))
    assert np.array_equal(q[in_segment], want8[in_segment]) and np.array_equal(codes[in_segment], want_codes[in_segment])
    a = torch.empty((rows, F), device="cuda")
    B.hm_gated(g_h, a)
    for pair, values in ((columns8, full), (a8, a)):
        got, got_codes = numbers8(pair)
        want8, want_codes, there = R.columns8(f64(values), offsets)
        places = np.repeat(there, 128)
        assert np.array_equal(got[:, places], want8[:, places]) and np.array_equal(got_codes[there], want_codes[there])
        assert is_poison(pair[0][:, torch.from_numpy(~places).cuda()]) and is_poison(pair[1][torch.from_numpy(~there).cuda()])


@pytest.mark.parametrize("F", [5, 128, 130, 768])
def test_each_output_alone_is_the_same(F):
    rows, counts = 300, [100, 0, 180]
    offsets = torch.tensor([0, 100, 100, 280], dtype=torch.int32, device="cuda")
    h, ga = drawn(1, rows, 2 * F, BF16, 2.0).cuda(), drawn(2, rows, F, BF16, 0.03).cuda()
    new = lambda: (torch.full((rows, 2 * F), 7.0, device="cuda"), *poisoned(B.alloc_rows8(rows, 2 * F)), *poisoned(B.alloc_columns8(rows, 3, 2 * F)),
                   *poisoned(B.alloc_columns8(rows, 3, F)))
    whole = new()
    B.hm_gated_backward(h, ga, offsets, *whole)
    for given in ((0,), (1, 2), (3, 4), (5, 6), (0, 1, 2), (0, 5, 6), (1, 2, 3, 4), (1, 2, 5, 6)):
        out = [t if i in given else None for i, t in enumerate(new())]
        B.hm_gated_backward(h, ga, offsets, *out)
        for i in given:
            assert torch.equal(out[i].view(torch.uint8), whole[i].view(torch.uint8)), (given, i)
    # without offsets every row
    free = [t if i < 3 else None for i, t in enumerate(new())]
    B.hm_gated_backward(h, ga, None, *free)
    for i in range(3):
        assert torch.equal(free[i][:280].view(torch.uint8), whole[i][:280].view(torch.uint8)) and not is_poison(free[i][280:])


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("F", [128, 130])
def test_what_is_no_number_becomes_nan_and_does_not_count(dtype, F):
    """Infinities and NaN in a block: those values are NaN in 8 bits, the others keep the scale that they have without them."""
    rows = 140
    h, ga = drawn(1, rows, 2 * F, dtype, 2.0), drawn(2, rows, F, dtype, 0.03)
    odd = torch.zeros((rows, F), dtype=torch.bool)
    for r, c, which, v in ((0, 0, "ga", float("inf")), (5, 77, "ga", float("-inf")), (9, 3, "ga", float("nan")), (127, 127, "gate", float("nan")),
                           (128, 2, "up", float("inf")), (130, 9, "up", float("nan")), (139, 100, "ga", float("inf"))):
        odd[r, c] = True
        if which == "ga":
            ga[r, c] = v
        else:
            h[r, c + (F if which == "up" else 0)] = v
    offsets = torch.tensor([0, rows], dtype=torch.int32, device="cuda")
    full, a = torch.empty((rows, 2 * F), device="cuda"), torch.empty((rows, F), device="cuda")
    rows8, a_rows8 = B.alloc_rows8(rows, 2 * F), B.alloc_rows8(rows, F)
    columns8, a8 = poisoned(B.alloc_columns8(rows, 1, 2 * F)), poisoned(B.alloc_columns8(rows, 1, F))
    B.hm_gated_backward(h.cuda(), ga.cuda(), offsets, full, *rows8, *columns8, *a8)
    B.hm_gated(h.cuda(), a, *a_rows8)
    finite = torch.isfinite(full).cpu()
    assert not finite[:, :F][odd].all() and finite[:, :F][~odd].all() and finite[:, F:][~odd].all()
    for pair, values in ((rows8, full), (a_rows8, a)):
        want, want_codes = R.rows8(f64(values))
        q, codes = numbers8(pair)
        assert np.array_equal(codes, want_codes) and np.array_equal(q, want, equal_nan=True)
    for pair, values in ((columns8, full), (a8, a)):
        want, want_codes, there = R.columns8(f64(values), offsets.cpu().numpy())
        q, codes = numbers8(pair)
        assert np.array_equal(codes[there], want_codes[there])
        assert np.array_equal(q[:, np.repeat(there, 128)], want[:, np.repeat(there, 128)], equal_nan=True)


def test_rows_of_segments_only():
    h = drawn(1, 40, 64, F32).cuda()
    offsets = torch.tensor([3, 3, 20, 31], dtype=torch.int32, device="cuda")
    a, pair = torch.full((40, 32), 7.0, device="cuda"), poisoned(B.alloc_rows8(40, 32))
    B.hm_gated(h, a, *pair, offsets=offsets)
    want = torch.empty((40, 32), device="cuda")
    B.hm_gated(h, want)
    assert torch.equal(a[3:31], want[3:31]) and bool((a[:3] == 7).all()) and bool((a[31:] == 7).all())
    assert is_poison(pair[0][:3]) and is_poison(pair[0][31:]) and is_poison(pair[1][31:]) and not is_poison(pair[0][3:31])


def test_offsets_that_make_no_sense_stay_inside():
    """Descending ones and ones beyond the rows: no access leaves the buffers; nothing is said about the results."""
    rows, F = 200, 128
    h, ga = drawn(1, rows, 2 * F, BF16).cuda(), drawn(2, rows, F, BF16).cuda()
    for bad in ([0, 500, 100, -7], [-5, 1 << 30, 3, 2], [150, 20, 10, 200], [300, 300, 300, 300]):
        offsets = torch.tensor(bad, dtype=torch.int32, device="cuda")
        B.hm_gated(h, torch.empty((rows, F), device="cuda"), *B.alloc_rows8(rows, F), offsets=offsets)
        B.hm_gated_backward(h, ga, offsets, torch.empty((rows, 2 * F), device="cuda"), *B.alloc_rows8(rows, 2 * F), *B.alloc_columns8(rows, 3, 2 * F),
                            *B.alloc_columns8(rows, 3, F))
    torch.cuda.synchronize()


def test_the_ways_through_a_graph_agree():
    rows, F = 300, 130
    h, ga = drawn(1, rows, 2 * F, BF16).cuda(), drawn(2, rows, F, BF16).cuda()
    offsets = torch.tensor([0, 120, 300], dtype=torch.int32, device="cuda")
    a, a8 = torch.empty((rows, F), dtype=BF16, device="cuda"), B.alloc_rows8(rows, F)
    outputs = (torch.empty((rows, 2 * F), dtype=BF16, device="cuda"), *B.alloc_rows8(rows, 2 * F), *poisoned(B.alloc_columns8(rows, 2, 2 * F)),
               *poisoned(B.alloc_columns8(rows, 2, F)))

    def step(stream=None):
        B.hm_gated(h, a, *a8, offsets, stream=stream)
        B.hm_gated_backward(h, ga, offsets, *outputs, stream=stream)
    every = [t.view(torch.uint8) for t in (a, *a8, *outputs)]
    step()
    want = [t.clone() for t in every]
    same = lambda: all(torch.equal(x, y) for x, y in zip(every, want))
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        step()
    torch.cuda.synchronize()
    assert same()
    step(side)
    torch.cuda.synchronize()
    assert same()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(3):
        for t in every[:6]:
            t.fill_(3)
        graph.replay()
        torch.cuda.synchronize()
        assert same()
        step()
        torch.cuda.synchronize()
        assert same()


def test_nothing_to_do_and_what_does_not_fit():
    e = lambda *shape, dtype=BF16: torch.zeros(shape, dtype=dtype, device="cuda")
    B.hm_gated(e(0, 64), e(0, 32))
    B.hm_gated_backward(e(0, 64), e(0, 32), gh=e(0, 64))
    h, ga, off = e(4, 64), e(4, 32), e(3, dtype=torch.int32)
    r8, c8, a8 = B.alloc_rows8(4, 32), B.alloc_columns8(4, 2, 64), B.alloc_columns8(4, 2, 32)
    gated = lambda **k: B.hm_gated(**{**dict(h=h, a=e(4, 32), q=r8[0], scale=r8[1], offsets=off), **k})
    back = lambda **k: B.hm_gated_backward(**{**dict(h=h, ga=ga, offsets=off, gh=e(4, 64), q_columns=c8[0], scale_columns=c8[1], a_columns=a8[0],
                                                     a_scale=a8[1]), **k})
    gated(), back()
    for bad in (dict(h=e(4, 63)), dict(a=e(4, 31)), dict(a=None, q=None, scale=None), dict(q=None), dict(scale=None), dict(q=r8[0][:3]), dict(h=e(64))):
        with pytest.raises(ValueError):
            gated(**bad)
    for bad in (dict(h=e(4, 64, dtype=torch.float16)), dict(a=e(4, 64)[:, :32]), dict(offsets=e(3, dtype=torch.int64)), dict(q=e(4, 128))):
        with pytest.raises(TypeError):
            gated(**bad)
    for bad in (dict(ga=e(3, 32)), dict(gh=e(4, 63)), dict(offsets=None), dict(scale_columns=None), dict(a_columns=None), dict(q_columns=c8[0][:, :128]),
                dict(gh=None, q_columns=None, scale_columns=None, a_columns=None, a_scale=None), dict(offsets=e(9, dtype=torch.int32))):
        with pytest.raises(ValueError):
            back(**bad)
    for bad in (dict(ga=e(4, 32, dtype=F32)), dict(gh=e(4, 64, dtype=torch.float16)), dict(ga=e(32, 4).t())):
        with pytest.raises(TypeError):
            back(**bad)


def test_offsets_of_no_entries_are_refused():
    """With and without a given stream, so by both halves of the binding; nothing is written."""
    h, ga, off = torch.ones((4, 64), device="cuda"), torch.ones((4, 32), device="cuda"), torch.zeros(0, dtype=torch.int32, device="cuda")
    for stream in (None, torch.cuda.current_stream()):
        a, gh, rows8 = torch.full((4, 32), 7.0, device="cuda"), torch.full((4, 64), 7.0, device="cuda"), poisoned(B.alloc_rows8(4, 64))
        with pytest.raises(ValueError, match="offsets"):
            B.hm_gated(h, a, offsets=off, stream=stream)
        with pytest.raises(ValueError, match="offsets"):
            B.hm_gated_backward(h, ga, off, gh, *rows8, stream=stream)
        with pytest.raises(B.HierMoEError):
            B.hm_gated(h, a, offsets=torch.zeros(1, dtype=torch.int32, device="cuda"), stream=stream)
        assert bool((a == 7).all()) and bool((gh == 7).all()) and all(is_poison(t) for t in rows8)
