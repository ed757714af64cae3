"""Refusals of the norm's, the activation's and the few tokens' calls, which need no GPU: nothing is launched; and the references
the GPU tests hold them to, by differences."""
import ctypes

import numpy as np
import pytest
import torch

import around_reference as A
from paper_2508_09591_amd import binding as B

fake_pointers = pytest.mark.skipif(torch.cuda.is_available(), reason="passes made-up device pointers: CPU-only by design")
P = lambda at=0x1000: ctypes.c_void_p(at)
BF16, F32 = B.HM_BF16, B.HM_F32


def refused(call, code, *cases):
    for bad in cases:
        assert call(**bad) == code, bad


@fake_pointers
def test_the_norm_checks_its_arguments():
    def call(x=P(), dtype=BF16, ld=64, res=P(), tdtype=BF16, rld=64, w=P(), wdtype=F32, eps=1e-6, rows=4, C=64, total=P(), tld=64, y=P(),
             ydtype=BF16, q=P(), s=P()):
        return B.lib().hm_rms_norm(x, dtype, ld, res, tdtype, rld, w, wdtype, eps, rows, C, total, tld, y, ydtype, q, s, None)

    refused(call, B.HM_ERR_NULL, dict(x=None), dict(w=None), dict(res=None), dict(total=None), dict(q=None), dict(s=None), dict(y=None, q=None, s=None))
    refused(call, B.HM_ERR_SHAPE, dict(dtype=2), dict(tdtype=2), dict(wdtype=-1), dict(ydtype=9), dict(rows=-1), dict(rows=1 << 31), dict(C=0),
            dict(C=32769), dict(eps=-1e-9), dict(eps=float("nan")), dict(ld=63), dict(rld=63), dict(tld=63), dict(x=P(0x1001)), dict(res=P(0x1001)),
            dict(total=P(0x1003)), dict(w=P(0x1002)), dict(y=P(0x1001)), dict(ydtype=F32, y=P(0x1002)), dict(q=P(0x1008)), dict(s=P(0x1002)))
    assert call(rows=0) == B.HM_OK
    assert call(rows=0, ld=1) == B.HM_OK


@fake_pointers
def test_the_norm_backward_checks_its_arguments():
    L = B.lib()

    def call(gy=P(), gdtype=BF16, gld=64, s=P(), dtype=BF16, sld=64, w=P(), wdtype=F32, eps=1e-6, rows=4, C=64, gt=P(), gtld=64, gx=P(), gxld=64,
             gw=P(), ws=P(), bytes=1 << 20):
        return L.hm_rms_norm_backward(gy, gdtype, gld, s, dtype, sld, w, wdtype, eps, rows, C, gt, gtld, gx, gxld, gw, ws, bytes, None)

    refused(call, B.HM_ERR_NULL, dict(gy=None), dict(s=None), dict(w=None), dict(gx=None), dict(gw=None))
    refused(call, B.HM_ERR_SHAPE, dict(gdtype=2), dict(dtype=3), dict(wdtype=-1), dict(rows=-1), dict(rows=1 << 31), dict(C=0), dict(C=32769),
            dict(eps=-1.0), dict(eps=float("nan")), dict(gld=63), dict(sld=1), dict(gtld=63), dict(gxld=0), dict(gy=P(0x1001)), dict(s=P(0x1001)),
            dict(w=P(0x1002)), dict(gt=P(0x1001)), dict(gx=P(0x1001)), dict(gw=P(0x1002)))
    need = L.hm_rms_norm_backward_workspace_bytes(4, 64)
    assert need > 0
    refused(call, B.HM_ERR_WORKSPACE, dict(ws=None), dict(bytes=need - 1), dict(ws=P(0x1008)))
    size = L.hm_rms_norm_backward_workspace_bytes
    assert size(-1, 8) == size(4, 0) == size(4, 32769) == 0 and size(0, 8) == size(1, 8) == 0
    assert max(size(n, 32768) for n in (2, 100, 10000, 1 << 30)) <= 512 * 32768 * 4


@fake_pointers
def test_the_activation_checks_its_arguments():
    L = B.lib()

    def call(h=P(), dtype=BF16, ld=64, off=P(), segments=2, rows=4, F=32, a=P(), adtype=BF16, q=P(), s=P()):
        return L.hm_gated(h, dtype, ld, off, segments, rows, F, a, adtype, q, s, None)

    def back(h=P(), ga=P(), dtype=BF16, ld=64, gld=32, off=P(), segments=2, rows=4, F=32, gh=P(), ghdtype=BF16, q=P(), s=P(), qc=P(), sc=P(), ac=P(),
             asc=P()):
        return L.hm_gated_backward(h, ga, dtype, ld, gld, off, segments, rows, F, gh, ghdtype, q, s, qc, sc, ac, asc, None)

    refused(call, B.HM_ERR_NULL, dict(h=None), dict(q=None), dict(s=None), dict(a=None, q=None, s=None))
    refused(back, B.HM_ERR_NULL, dict(h=None), dict(ga=None), dict(q=None), dict(s=None), dict(qc=None), dict(sc=None), dict(ac=None), dict(asc=None),
            dict(gh=None, q=None, s=None, qc=None, sc=None, ac=None, asc=None), dict(off=None), dict(off=None, ac=None, asc=None),
            dict(off=None, qc=None, sc=None))
    for f in (call, back):
        refused(f, B.HM_ERR_SHAPE, dict(dtype=2), dict(F=0), dict(rows=-1), dict(rows=1 << 31), dict(segments=0), dict(segments=1025),
                dict(rows=(1 << 31) - 200), dict(ld=63), dict(h=P(0x1001)), dict(q=P(0x1004)), dict(s=P(0x1001)), dict(off=P(0x1002)),
                dict(rows=1 << 30, F=4096))
        assert f(rows=0) == B.HM_OK
    refused(call, B.HM_ERR_SHAPE, dict(F=(1 << 20) + 1, ld=1 << 23), dict(adtype=4), dict(a=P(0x1001)), dict(off=None, rows=(1 << 25) + 1, F=512, ld=1024))
    refused(back, B.HM_ERR_SHAPE, dict(F=(1 << 19) + 1, ld=1 << 23, gld=1 << 23), dict(gld=31), dict(ga=P(0x1001)), dict(ghdtype=4), dict(gh=P(0x1001)),
            dict(qc=P(0x1004)), dict(sc=P(0x1001)), dict(ac=P(0x1008)), dict(asc=P(0x1002)),
            dict(off=None, rows=(1 << 25) + 1, F=256, ld=512, gld=256, qc=None, sc=None, ac=None, asc=None),
            dict(ld=(1 << 22) + 1), dict(gld=(1 << 22) + 1))   # with columns


@fake_pointers
def test_the_layer_of_a_few_tokens_checks_its_arguments():
    L = B.lib()

    def call(x=P(), ld=64, logits=P(), ldtype=F32, lld=64, bias=None, T=4, E=64, K=4, groups=1, w13=P(), s13=P(), w2=P(), s2=P(), first=0, experts=8,
             H=64, F=32, ids=P(), weights=P(), out=P(), odtype=BF16, ws=P(), bytes=1 << 20, router=True):
        r = ctypes.byref(B.hm_router(E, K, 0, groups, 1, 1, 1, 1.0)) if router else None
        return L.hm_layer_few(x, ld, logits, ldtype, lld, bias, T, r, w13, s13, w2, s2, first, experts, H, F, ids, weights, out, odtype, ws, bytes, None)

    refused(call, B.HM_ERR_NULL, *[{n: None} for n in ("x", "logits", "w13", "s13", "w2", "s2", "ids", "weights", "out")], dict(router=False))
    refused(call, B.HM_ERR_SHAPE, dict(T=-1), dict(T=65), dict(K=0), dict(K=65), dict(K=17, T=61), dict(E=0), dict(E=4097, lld=4097), dict(groups=3),
            dict(first=-1), dict(first=57), dict(experts=0), dict(experts=65), dict(experts=1025, E=2048, lld=2048), dict(H=0), dict(H=(1 << 20) + 1, ld=1 << 21),
            dict(F=0), dict(F=(1 << 19) + 1), dict(ld=63), dict(lld=63), dict(ldtype=2), dict(odtype=2), dict(x=P(0x1001)), dict(out=P(0x1001)),
            dict(out=P(0x1002), odtype=F32), dict(w13=P(0x1008)), dict(w2=P(0x1004)), dict(s13=P(0x1001)), dict(s2=P(0x1002)),
            dict(T=64, K=16, experts=1024, E=1024, lld=1024, F=1 << 19))
    need = L.hm_layer_few_workspace_bytes(4, 4, 64, 32)
    refused(call, B.HM_ERR_WORKSPACE, dict(ws=None), dict(bytes=need - 1), dict(ws=P(0x1004)))
    assert call(T=0, x=None, w13=None, ws=None, out=None) == B.HM_OK
    size = L.hm_layer_few_workspace_bytes
    assert size(65, 1, 8, 8) == size(-1, 1, 8, 8) == size(1, 0, 8, 8) == size(64, 17, 8, 8) == 0
    assert size(1, 1, 8, 0) == size(1, 1, 8, (1 << 19) + 1) == size(1, 1, 0, 8) == size(1, 1, (1 << 20) + 1, 8) == 0
    assert need > 0 and size(64, 16, 1 << 20, 1 << 19) == 1024 * (6 * (1 << 19) + 4 * (1 << 20))


def test_the_binding_says_what_does_not_fit():
    z = lambda *shape, dtype=torch.bfloat16: torch.zeros(shape, dtype=dtype)
    r8 = lambda rows, C: B.alloc_rows8(rows, C, device="cpu")
    x, w, f32 = z(4, 64), z(64, dtype=torch.float32), torch.float32
    with pytest.raises(TypeError, match="no CPU path"):
        B.hm_rms_norm(x, w, 1e-6, z(4, 64))
    with pytest.raises(TypeError, match="no CPU path"):
        B.hm_rms_norm_backward(x, x, w, 1e-6, z(4, 64), z(64, dtype=f32))
    with pytest.raises(TypeError, match="no CPU path"):
        B.hm_gated(x, z(4, 32))
    with pytest.raises(TypeError, match="no CPU path"):
        B.hm_gated_backward(x, z(4, 32), gh=z(4, 64))
    with pytest.raises(TypeError, match="no CPU path"):
        B.hm_layer_few(x, z(4, 8), B.Router(8, 2), *B.alloc_weights8(8, 64, 64, device="cpu"), *B.alloc_weights8(8, 64, 32, device="cpu"),
                       z(4, 2, dtype=torch.int32), z(4, 2, dtype=f32), z(4, 64))


def test_offsets_of_no_entries_are_not_none():
    """They have no address, which the library takes for all rows."""
    i32 = lambda n: torch.zeros(n, dtype=torch.int32)
    assert B._segments(None) == 0 and B._segments(i32(2)) == 1 and B._segments(i32(17)) == 16
    assert B._segments(i32(1)) == 0   # which the library refuses, as there is an address
    with pytest.raises(ValueError, match="offsets"):
        B._segments(i32(0))


NAMES = [n[3:] for n in B._NATIVE_AROUND]


@pytest.mark.parametrize("name", NAMES)
def test_anything_out_of_the_ordinary_is_left_to_python(name):
    B.lib()
    f = getattr(B._native, name)
    cpu = torch.zeros((4, 8), dtype=torch.bfloat16)
    for n in range(18):
        for arg in (None, 1, 1.5, "x", [1, 2], cpu, torch.zeros((4, 8), dtype=torch.float32, device="meta")):
            assert f(*[arg] * n) is None
    with pytest.raises(TypeError):
        B._native.bind_around(1, 2)


# ---- the references, by differences ---------------------------------------------------------------------------------
def differences(f, x, g, h=1e-6):
    """Gradient of sum(f(x) g) by central differences."""
    out = np.zeros_like(x)
    for i in np.ndindex(x.shape):
        a, b = x.copy(), x.copy()
        a[i] += h
        b[i] -= h
        out[i] = ((f(a) - f(b)) * g).sum() / (2 * h)
    return out


def test_the_gradients_of_the_references():
    rng = np.random.default_rng(3)
    s, w, gy, gt = rng.standard_normal((3, 7)), 1 + 0.1 * rng.standard_normal(7), rng.standard_normal((3, 7)), rng.standard_normal((3, 7))
    gx, _, gw, _ = A.rms_norm_backward(gy, s, w, 1e-3, gt, 1)
    assert np.abs(gx - gt - differences(lambda v: A.rms_norm(v, w, 1e-3)[0], s, gy)).max() < 1e-8
    assert np.abs(gw - differences(lambda v: A.rms_norm(s, v, 1e-3)[0], w, gy)).max() < 1e-8
    h, ga = 2 * rng.standard_normal((3, 10)), rng.standard_normal((3, 5))
    assert np.abs(A.gated_backward(h, ga)[0] - differences(lambda v: A.gated(v)[0], h, ga)).max() < 1e-8
