"""Refusals of the router's and the experts' calls, which need no GPU: nothing is launched."""
import ctypes

import pytest
import torch

from paper_2508_09591_amd import binding as B

fake_pointers = pytest.mark.skipif(torch.cuda.is_available(), reason="passes made-up device pointers: CPU-only by design")
P = lambda at=0x1000: ctypes.c_void_p(at)


def router(E=64, K=4, score=0, groups=1, top=1, best=1):
    return ctypes.byref(B.hm_router(E, K, score, groups, top, best, 1, 1.0))


BAD_ROUTERS = [dict(E=0), dict(E=4097), dict(K=0), dict(K=65), dict(score=2), dict(score=-1), dict(groups=0), dict(groups=3), dict(groups=65),
               dict(groups=4, top=5), dict(groups=4, top=0), dict(best=0), dict(best=3), dict(E=8, K=1, groups=8, best=2), dict(E=8, K=3, groups=4, top=1),
               dict(E=3, K=4)]


@fake_pointers
def test_the_router_is_refused_what_it_cannot_do():
    L = B.lib()

    def route(logits=P(), dtype=B.HM_F32, ld=64, T=4, r=router(), ids=P(), w=P()):
        return L.hm_route(logits, dtype, ld, None, T, r, ids, w, None)

    def back(logits=P(), dtype=B.HM_F32, ld=64, ids=P(), g=P(), T=4, r=router(), out=P(), grad_ld=64):
        return L.hm_route_backward(logits, dtype, ld, ids, g, T, r, out, grad_ld, None)

    for call, pointers in ((route, ("logits", "ids", "w")), (back, ("logits", "ids", "g", "out"))):
        for name in pointers:
            assert call(**{name: None}) == B.HM_ERR_NULL
        assert call(r=None) == B.HM_ERR_NULL
        for bad in BAD_ROUTERS:
            assert call(r=router(**bad), ld=4097) == B.HM_ERR_SHAPE, bad
        assert call(T=-1) == B.HM_ERR_SHAPE and call(T=1 << 30) == B.HM_ERR_SHAPE
        assert call(dtype=2) == B.HM_ERR_SHAPE and call(ld=63) == B.HM_ERR_SHAPE
        assert call(T=0) == B.HM_OK
    assert back(grad_ld=63) == B.HM_ERR_SHAPE


@fake_pointers
def test_the_weights_gradient_checks_its_arguments():
    L, c = B.lib(), B.hm_plan_out()
    c.slot_row, c.status = 0x1000, 0x1000

    def call(gout=P(), y=P(), dtype=B.HM_BF16, y_rows=8, T=4, K=2, H=8, plan=c, out=P()):
        return L.hm_combine_weight_grad(gout, y, dtype, y_rows, T, K, H, None if plan is None else ctypes.byref(plan), out, None)

    for name in ("gout", "y", "plan", "out"):
        assert call(**{name: None}) == B.HM_ERR_NULL
    assert call(plan=B.hm_plan_out()) == B.HM_ERR_NULL
    for bad in (dict(T=-1), dict(K=0), dict(K=65), dict(H=0), dict(y_rows=-1), dict(dtype=7), dict(T=1 << 30, K=4)):
        assert call(**bad) == B.HM_ERR_SHAPE, bad
    assert call(T=0) == B.HM_OK


@fake_pointers
def test_quantising_checks_its_arguments():
    L = B.lib()
    rows = lambda x=P(), dtype=0, ld=64, rows=4, C=64, q=P(), s=P(): L.hm_quantize_rows(x, dtype, ld, rows, C, q, s, None)
    cols = lambda x=P(), dtype=0, ld=64, off=P(), segments=2, rows=4, C=64, q=P(), s=P(): L.hm_quantize_columns(x, dtype, ld, off, segments, rows, C, q, s, None)
    wts = lambda x=P(), dtype=0, E=2, N=4, C=64, q=P(), s=P(), qt=None, st=None: L.hm_quantize_weights(x, dtype, E, N, C, q, s, qt, st, None)
    for call in (rows, cols, wts):
        for name in ("x", "q", "s"):
            assert call(**{name: None}) == B.HM_ERR_NULL
        for bad in (dict(dtype=2), dict(C=0), dict(C=(1 << 20) + 1), dict(q=P(0x1008)), dict(s=P(0x1002))):
            assert call(**bad) == B.HM_ERR_SHAPE, bad
    for call in (rows, cols):
        for bad in (dict(ld=63), dict(rows=-1), dict(rows=1 << 31)):
            assert call(**bad) == B.HM_ERR_SHAPE, bad
        assert call(rows=0) == B.HM_OK
    assert cols(off=None) == B.HM_ERR_NULL
    for bad in (dict(segments=0), dict(segments=1025), dict(rows=(1 << 31) - 1 - 128)):
        assert cols(**bad) == B.HM_ERR_SHAPE, bad
    for bad in (dict(E=0), dict(E=1025), dict(N=0), dict(N=(1 << 20) + 1), dict(qt=P(0x1004), st=P()), dict(qt=P(), st=P(0x1001))):
        assert wts(**bad) == B.HM_ERR_SHAPE, bad
    assert wts(qt=P()) == B.HM_ERR_NULL and wts(st=P()) == B.HM_ERR_NULL


@fake_pointers
def test_products_check_their_arguments():
    L = B.lib()
    for fn in (L.hm_expert_matmul, L.hm_expert_matmul_dw):
        def call(a=P(), sa=P(), b=P(), sb=P(), off=P(), E=2, rows=4, N=8, H=16, out=P(), dtype=B.HM_BF16):
            return fn(a, sa, b, sb, off, E, rows, N, H, out, dtype, None)

        for name in ("a", "sa", "b", "sb", "off", "out"):
            assert call(**{name: None}) == B.HM_ERR_NULL
        for bad in (dict(E=0), dict(E=1025), dict(rows=-1), dict(rows=(1 << 31) - 128), dict(N=0), dict(N=(1 << 20) + 1), dict(H=0), dict(H=(1 << 20) + 1),
                    dict(a=P(0x1008)), dict(b=P(0x1004)), dict(sa=P(0x1001)), dict(sb=P(0x1002)), dict(out=P(0x1001)), dict(dtype=5),
                    dict(out=P(0x1002), dtype=B.HM_F32)):
            assert call(**bad) == B.HM_ERR_SHAPE, bad
    assert L.hm_expert_matmul(P(), P(), P(), P(), P(), 2, 0, 8, 16, P(), 0, None) == B.HM_OK
    assert L.hm_expert_matmul(P(), P(), P(), P(), P(), 1024, 1 << 25, 8, 16, P(), 0, None) == B.HM_ERR_SHAPE
    assert L.hm_expert_matmul(P(), P(), P(), P(), P(), 1, 1 << 30, 1 << 20, 16, P(), 0, None) == B.HM_ERR_SHAPE
    assert L.hm_expert_matmul_dw(P(), P(), P(), P(), P(), 1, 1 << 24, 8, 16, P(), 0, None) == B.HM_ERR_SHAPE


def test_the_binding_refuses_tensors_it_cannot_use():
    z = lambda *shape, dtype=torch.float32: torch.zeros(shape, dtype=dtype)
    r = B.Router(8, 2)
    ids, w = z(4, 2, dtype=torch.int32), z(4, 2)
    with pytest.raises(TypeError, match="no CPU path"):
        B.hm_route(z(4, 8), r, ids, w)
    with pytest.raises(TypeError, match="no CPU path"):
        B.hm_quantize_rows(z(4, 8), *B.alloc_rows8(4, 8, device="cpu"))
    with pytest.raises(TypeError, match="no CPU path"):
        B.hm_expert_matmul(*B.alloc_rows8(4, 8, device="cpu"), *B.alloc_weights8(2, 4, 8, device="cpu"), z(3, dtype=torch.int32), z(4, 4))
    with pytest.raises(ValueError, match="softmax or sigmoid"):
        B.Router(8, 2, "tanh")


@pytest.mark.parametrize("width", [0, 1, 100, 127, 129, 300])
def test_products_take_whole_blocks_of_values(width):
    """The kernels read blocks of 128: operands that do not hold them whole are refused, whatever else fits."""
    e8 = lambda *shape: torch.zeros(shape, dtype=torch.float8_e4m3fn)
    byte = lambda *shape: torch.zeros(shape, dtype=torch.uint8)
    operands = (e8(4, width), byte(4, B.scale8_bytes(width)), e8(2, 8, width), byte(2, 1, B.scale8_bytes(width)))
    with pytest.raises(ValueError, match="whole blocks"):
        B.hm_expert_matmul(*operands, torch.zeros(3, dtype=torch.int32), torch.zeros((4, 8)))


def test_sizes_of_the_layouts():
    assert [B.row8_bytes(c) for c in (1, 128, 129, 7168)] == [128, 128, 256, 7168]
    assert [B.scale8_bytes(c) for c in (1, 512, 513, 7168)] == [4, 4, 8, 56]
    q, s = B.alloc_columns8(300, 3, 70, device="cpu")
    assert tuple(q.shape) == (70, 128 * 5) and tuple(s.shape) == (5, 70)
    q, s = B.alloc_weights8(2, 130, 600, device="cpu")
    assert tuple(q.shape) == (2, 130, 640) and tuple(s.shape) == (2, 2, 8)
