"""hm_rms_norm and its way back against 64-bit references."""
import numpy as np
import pytest
import torch

import around_reference as A
import layer_reference as R
from paper_2508_09591_amd import binding as B

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32
KIND = {BF16: "bf16", F32: "f32"}
EPS = 1e-6


def drawn(seed, rows, C, dtype, sigma=1.0):
    """Rows of many sizes on the CPU, exactly as the kernel reads them."""
    g = torch.Generator()
    g.manual_seed(seed)
    x = torch.randn((rows, C), generator=g) * torch.exp(2 * torch.randn((rows, 1), generator=g)) * sigma
    return x.to(dtype)


def spaced(t, extra):
    """The matrix on the GPU with rows `extra` elements further apart, off a vector's alignment where that is odd, NaN between."""
    rows, C = t.shape
    m = torch.full((rows * (C + extra) + extra,), float("nan"), dtype=t.dtype, device="cuda")[extra:].view(rows, C + extra)[:, :C]
    return m.copy_(t)


def untouched(m):
    """Whether what lies between a spaced matrix's rows is still NaN."""
    rows, gap = m.shape[0], m.stride(0) - m.shape[1]
    between = torch.as_strided(m, (rows - 1, gap), (m.stride(0), 1), m.storage_offset() + m.shape[1]) if rows > 1 else torch.empty(0)
    return bool(torch.isnan(between).all())


def f64(t):
    return t.double().cpu().numpy()


def numbers8(q, s):
    return q.float().cpu().numpy().astype(np.float64), s.view(torch.uint8).cpu().numpy()


SIZES = [(1, 1), (1, 7168), (3, 7), (5, 127), (2, 129), (9, 511), (4, 512), (66, 513), (7, 1030), (3, 2056), (5, 2049), (3, 4100), (4, 8192), (3, 8200), (2, 16390),
         (2, 32768), (1, 32761), (600, 1000), (520, 4200)]
TYPES = [(BF16, None, F32), (BF16, BF16, BF16), (BF16, F32, F32), (F32, None, BF16), (F32, F32, F32), (F32, BF16, F32)]


@pytest.mark.parametrize("dtype,kept,wtype", TYPES)
@pytest.mark.parametrize("rows,C", SIZES)
def test_norm(rows, C, dtype, kept, wtype):
    x = drawn(rows + C, rows, C, dtype)
    r = None if kept is None else drawn(rows + C + 1, rows, C, kept)
    w = (1 + 0.1 * drawn(7, 1, C, F32)[0]).to(wtype)
    s = x if r is None else (x.float() + r.float()).to(kept)
    want, off = A.rms_norm(f64(s), f64(w), EPS)
    for extra, ytype in ((0, BF16), (8, F32), (3, F32)):
        gx, gr = spaced(x, extra), None if r is None else spaced(r, extra)
        total = None if r is None else spaced(torch.zeros_like(r), extra)
        y, (q, scale) = torch.full((rows, C), float("nan"), dtype=ytype, device="cuda"), B.alloc_rows8(rows, C)
        B.hm_rms_norm(gx, w.cuda(), EPS, y, q, scale, gr, total)
        if r is not None:
            assert torch.equal(total.cpu(), s) and untouched(total)
        assert (np.abs(f64(y) - want) <= A.HALF[KIND[ytype]] * (np.abs(want) + off) + off + A.TINY).all()
        values, codes = numbers8(q, scale)
        A.check_rows8(values, codes, want, off)
        if ytype == F32:   # the same values, rounded once
            want8, want_codes = R.rows8(f64(y))
            assert np.array_equal(values, want8) and np.array_equal(codes.astype(np.int64), want_codes)
        alone, only = torch.empty_like(y), B.alloc_rows8(rows, C)   # one output without the other: the same bits
        B.hm_rms_norm(gx, w.cuda(), EPS, alone, None, None, gr, total)
        B.hm_rms_norm(gx, w.cuda(), EPS, None, *only, gr, total)
        assert torch.equal(alone, y) and all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(only, (q, scale)))


def test_many_rows_and_rows_in_place():
    """More rows than a launch has workgroups; the sum in the residual's place, y in x's."""
    for rows, C in ((9001, 520), (5003, 2056)):
        x, r, w = drawn(1, rows, C, BF16), drawn(2, rows, C, BF16), torch.ones(C)
        s = (x.float() + r.float()).to(BF16)
        want, off = A.rms_norm(f64(s), f64(w), EPS)
        gx, gr = x.cuda(), r.cuda()
        B.hm_rms_norm(gx, w.cuda(), EPS, gx, None, None, gr, gr)
        assert torch.equal(gr.cpu(), s)
        assert (np.abs(f64(gx) - want) <= A.HALF["bf16"] * (np.abs(want) + off) + off).all()
        other = x.cuda()
        B.hm_rms_norm(other, w.cuda(), EPS, other)   # no residual
        want, off = A.rms_norm(f64(x), f64(w), EPS)
        assert (np.abs(f64(other) - want) <= A.HALF["bf16"] * (np.abs(want) + off) + off).all()


def test_rows_that_are_no_numbers():
    """Zeros give zeros, a NaN its own row only, as values and in 8 bits."""
    x = drawn(3, 6, 300, F32)
    x[1] = 0.0
    x[2, 17] = float("nan")
    x[3, 299] = float("inf")
    x[4] = 1e-30
    y, (q, s) = torch.empty((6, 300), device="cuda"), B.alloc_rows8(6, 300)
    B.hm_rms_norm(x.cuda(), torch.ones(300, device="cuda"), EPS, y, q, s)
    assert not y[1].any() and torch.isnan(y[2]).all() and torch.isnan(q[2].float()[:300]).all() and not q.float()[1].any()
    assert torch.isnan(y[3, 299]) and not y[3, :299].any()   # inf / inf, and finite numbers over inf
    want, off = A.rms_norm(x[[0, 4, 5]].double().numpy(), np.ones(300), EPS)
    assert (np.abs(f64(y[[0, 4, 5]]) - want) <= A.U * np.abs(want) + off + A.TINY).all()


@pytest.mark.parametrize("rows,C", [(512, 1030), (1024, 1000), (448, 40)])
def test_the_weights_gradient_keeps_small_parts_beside_large_ones(rows, C):
    """A row a part, whose terms are exact: 1, and many of 2^-25, of which fp32 keeps none beside the 1.  64 sums of fp32 have up to
    rows / 64 + 3 parts each, half a step of 1 for every addition, and are added up in 64 bits and rounded once; one sum of a 16th of the
    parts would lose rows / 32 - 1/2 half steps."""
    assert parts_of(rows, C) == rows
    gy = torch.full((rows, C), 2.0 ** -25, device="cuda")
    gy[0] = 1.0
    s, gw = torch.ones_like(gy), torch.empty(C, device="cuda")
    B.hm_rms_norm_backward(gy, s, torch.ones(C, device="cuda"), 0.0, torch.empty_like(gy), gw)
    want = 1.0 + (rows - 1) * 2.0 ** -25
    assert rows / 64 + 4 < rows / 32 - 0.5
    assert (np.abs(f64(gw) - want) <= (rows / 64 + 4) * A.U * want).all()


def test_no_rows():
    w = torch.ones(64, device="cuda")
    none, gw = torch.empty((0, 64), dtype=BF16, device="cuda"), torch.full((64,), 5.0, device="cuda")
    B.hm_rms_norm(none, w, EPS, none)
    B.hm_rms_norm_backward(none, none, w, EPS, none, gw)
    assert not gw.any()


def parts_of(rows, C):
    bytes_ = int(B.lib().hm_rms_norm_backward_workspace_bytes(rows, C))
    return max(bytes_ // (4 * C), 1)


@pytest.mark.parametrize("gtype,dtype,wtype,past", [(BF16, BF16, F32, True), (BF16, BF16, BF16, False), (BF16, F32, F32, True), (F32, F32, F32, False),
                                                    (F32, BF16, BF16, True), (F32, F32, BF16, True)])
@pytest.mark.parametrize("rows,C", SIZES + [(1237, 1030), (2100, 72), (700, 2056)])
def test_norm_backward(rows, C, gtype, dtype, wtype, past):
    s, gy = drawn(rows + C, rows, C, dtype), drawn(rows + C + 1, rows, C, gtype, 0.03)
    gt = drawn(rows + C + 2, rows, C, dtype, 0.03) if past else None
    w = (1 + 0.1 * drawn(7, 1, C, F32)[0]).to(wtype)
    gx, off, gw, off_w = A.rms_norm_backward(f64(gy), f64(s), f64(w), EPS, None if gt is None else f64(gt), parts_of(rows, C))
    for extra in (0, 3):
        to, to_w = spaced(torch.zeros_like(s), extra), torch.full((C,), float("nan"), device="cuda")
        workspace = B.alloc_rms_norm_workspace(rows, C).fill_(0xAB)
        B.hm_rms_norm_backward(spaced(gy, extra), spaced(s, extra), w.cuda(), EPS, to, to_w, None if gt is None else spaced(gt, extra), workspace)
        assert (np.abs(f64(to) - gx) <= A.HALF[KIND[dtype]] * (np.abs(gx) + off) + off + A.TINY).all() and untouched(to)
        assert (np.abs(f64(to_w) - gw) <= off_w + A.TINY).all()
    if past:   # in the gradient's own place
        here, again = gt.cuda(), torch.empty_like(to_w)
        B.hm_rms_norm_backward(gy.cuda(), s.cuda(), w.cuda(), EPS, here, again, here)
        assert torch.equal(here, to) and torch.equal(again, to_w)


def test_the_ways_through_a_graph_agree():
    """Captured and replayed, with eager calls between that share the workspace: the same bits each time."""
    rows, C = 600, 1030
    x, r, w, gy = drawn(1, rows, C, BF16).cuda(), drawn(2, rows, C, F32).cuda(), torch.ones(C, device="cuda"), drawn(3, rows, C, BF16, 0.03).cuda()
    total, y, (q, s) = torch.empty_like(r), torch.empty_like(x), B.alloc_rows8(rows, C)
    gx, gw, ws = torch.empty_like(r), torch.empty_like(w), B.alloc_rms_norm_workspace(rows, C)

    def step(stream=None):
        B.hm_rms_norm(x, w, EPS, y, q, s, r, total, stream=stream)
        B.hm_rms_norm_backward(gy, total, w, EPS, gx, gw, total, ws, stream=stream)
    outputs = (total, y, q.view(torch.uint8), s, gx, gw)
    step()
    want = [t.clone() for t in outputs]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        step()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(outputs, want))
    step(side)   # through ctypes
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(outputs, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(3):
        for t in outputs:
            t.fill_(7)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outputs, want))
        step()
        torch.cuda.synchronize()


def test_what_does_not_fit_is_refused():
    e = lambda *shape, dtype=BF16: torch.zeros(shape, dtype=dtype, device="cuda")
    x, w, ok8 = e(4, 64), e(64, dtype=F32), B.alloc_rows8(4, 64)
    norm = lambda **k: B.hm_rms_norm(**{**dict(x=x, weight=w, eps=EPS, y=e(4, 64), q=ok8[0], scale=ok8[1], residual=e(4, 64), total=e(4, 64)), **k})
    back = lambda **k: B.hm_rms_norm_backward(**{**dict(gy=x, s=x, weight=w, eps=EPS, gx=e(4, 64), gweight=e(64, dtype=F32), gtotal=e(4, 64)), **k})
    norm(), back()
    for bad in (dict(weight=e(63)), dict(y=e(4, 63)), dict(y=None, q=None, scale=None), dict(q=None), dict(scale=None), dict(residual=None), dict(total=None),
                dict(residual=e(5, 64)), dict(total=e(4, 65)), dict(q=e(4, 64, dtype=torch.uint8)), dict(x=e(64))):
        with pytest.raises(ValueError):
            norm(**bad)
    for bad in (dict(x=e(4, 64, dtype=torch.float16)), dict(total=e(4, 64, dtype=F32)), dict(x=e(64, 4).t()), dict(weight=e(128)[::2]), dict(y=e(4, 128)[:, :64]),
                dict(y=e(4, 64, dtype=torch.float64))):
        with pytest.raises((TypeError, ValueError)):
            norm(**bad)
    for bad in (dict(gy=e(3, 64)), dict(gx=e(4, 65)), dict(gweight=e(65, dtype=F32)), dict(gtotal=e(5, 64)), dict(weight=e(63))):
        with pytest.raises(ValueError):
            back(**bad)
    for bad in (dict(gx=e(4, 64, dtype=F32)), dict(gtotal=e(4, 64, dtype=F32)), dict(gweight=e(64)), dict(gy=e(4, 64, dtype=torch.float16))):
        with pytest.raises(TypeError):
            back(**bad)
    with pytest.raises(B.HierMoEError):
        back(workspace=e(8, dtype=torch.uint8))
    with pytest.raises(B.HierMoEError):
        norm(eps=-1.0)
