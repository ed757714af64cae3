"""A mixture-of-experts layer on one rank, forward and backward, out of the library's calls: an example of how they go
together.

Norm with the residual's addition, router, plan, dispatch, the experts' products in 8 bits with the activation between
them, combine; up to 64 experts, all of them here (an exchange between ranks would stand behind the dispatch and before the
combine).  An expert is w2 (silu(gate) * up) with gate and up from one product with w13.  Up to 64 tokens may go through
few(), without a plan.  PyTorch does what the library has no call for: the router's own product, and the memory.

    python -m paper_2508_09591_amd.layer        # times a forward and a backward pass on the current GPU
"""
from __future__ import annotations

import time

import torch

from . import binding as hm


class ExpertLayer:
    """gate [E, H] fp32; w13 [E, 2 F, H] and w2 [E, H, F], bf16 or fp32: the master weights, H a multiple of 512 (so
    that rows of 8 bits and their scales are rows of 2-byte units).  quantize() lays the weights out in 8 bits, both
    ways round: call it again after an optimizer step.  forward() keeps what backward() needs.  gone [E], bool: experts
    that no token may choose, say those of a rank that is lost: their logits are -inf and their gradients 0, while the
    gate stays finite.  It may be set between passes.  norm [H]: the weight of a norm in front of the layer, which then
    takes x + residual; the last call's sum is self.total."""

    def __init__(self, gate: torch.Tensor, w13: torch.Tensor, w2: torch.Tensor, router: hm.Router, bias=None,
                 gone=None, norm=None, eps: float = 1e-6):
        self.gate, self.w13, self.w2, self.router, self.bias, self.gone = gate, w13, w2, router, bias, gone
        self.norm, self.eps = norm, eps
        self.E, self.H, self.F = w2.shape
        if self.E != router.E or self.E > 64 or self.H % 512:
            raise ValueError("at most 64 experts, as many as the router's, and rows of a multiple of 512 values")
        # every expert is a destination of its own
        self.dest = torch.arange(self.E, dtype=torch.int32, device=w2.device)
        self.quantize()

    def quantize(self):
        both = lambda w: hm.hm_quantize_weights(w, *hm.alloc_weights8(*w.shape, device=w.device),
                                                *hm.alloc_weights8(w.shape[0], w.shape[2], w.shape[1], device=w.device))
        w13, w2 = both(self.w13), both(self.w2)
        self.q13, self.q13_t, self.q2, self.q2_t = w13[:2], w13[2:], w2[:2], w2[2:]

    def _rows8(self, x):
        return hm.hm_quantize_rows(x, *hm.alloc_rows8(*x.shape, device=x.device))

    def _columns8(self, x):
        return hm.hm_quantize_columns(x, self.plan.dest_offset, *self._alloc_columns8(x.shape[1], x.device))

    def _alloc_columns8(self, columns, device):
        return hm.alloc_columns8(self.rows, self.E, columns, device=device)

    def _product(self, x8, w8, columns):
        out = torch.empty((x8[0].shape[0], columns), dtype=torch.bfloat16, device=x8[0].device)
        return hm.hm_expert_matmul(*x8, *w8, self.plan.dest_offset, out)

    def _spread(self, rows):
        """Rows of bytes to the experts' rows: a dispatch copies 2-byte units, whatever they mean."""
        units = rows.view(torch.bfloat16)
        out = torch.zeros((self.rows, units.shape[1]), dtype=torch.bfloat16, device=rows.device)
        return hm.hm_dispatch_pack(units, self.plan, out).view(rows.dtype)

    def _normed(self, x, residual, rows8: bool):
        """What the router and the experts take, and the same in 8 bits if it is wanted; without a norm x itself."""
        if self.norm is None:
            if residual is not None:
                raise ValueError("a residual goes with a norm")
            return x, self._rows8(x) if rows8 else None
        self.total = x if residual is None else torch.empty_like(residual)
        y, q, scale, _ = hm.hm_rms_norm(x, self.norm, self.eps, torch.empty_like(x),
                                        *(hm.alloc_rows8(*x.shape, device=x.device) if rows8 else (None, None)), residual,
                                        None if residual is None else self.total)
        return y, (q, scale)

    def _logits(self, x):
        logits = x.float() @ self.gate.t()
        return logits if self.gone is None else logits.masked_fill_(self.gone, float("-inf"))

    def few(self, x: torch.Tensor, residual=None) -> torch.Tensor:
        """forward() for up to 64 tokens that nothing is learnt from: what is between the products is not rounded to 8
        bits, and nothing is kept for backward()."""
        T, K = x.shape[0], self.router.K
        x, _ = self._normed(x, residual, False)
        empty = lambda dtype: torch.empty((T, K), dtype=dtype, device=x.device)
        return hm.hm_layer_few(x, self._logits(x), self.router, *self.q13, *self.q2, empty(torch.int32), empty(torch.float32),
                               torch.empty_like(x), bias=self.bias)

    def forward(self, x: torch.Tensor, residual=None) -> torch.Tensor:
        """x [T, H] bf16 -> [T, H] bf16."""
        T, K = x.shape[0], self.router.K
        x, x8 = self._normed(x, residual, True)   # in 8 bits once a token, then half the bytes to spread
        self.x, self.logits = x, self._logits(x)
        self.normed = None if self.norm is None else self.total   # few() in between has a total of its own
        self.ids = torch.empty((T, K), dtype=torch.int32, device=x.device)
        self.weights = torch.empty((T, K), dtype=torch.float32, device=x.device)
        hm.hm_route(self.logits, self.router, self.ids, self.weights, self.bias)
        # one row for every slot, ordered by expert; slots the router dropped leave the last rows unused
        self.plan = hm.alloc_plan(T, K, self.E, 1, 1, hm.HM_DEDUP_NONE, num_dest=self.E, device=x.device)
        self.rows = T * K
        hm.hm_plan_mapped(self.ids, self.weights, self.dest, self.E, False, plan=self.plan)
        self.h = self._product((self._spread(x8[0]), self._spread(x8[1])), self.q13, 2 * self.F)
        _, *a8 = hm.hm_gated(self.h, None, *hm.alloc_rows8(self.rows, self.F, device=x.device), self.plan.dest_offset)
        self.y = self._product(a8, self.q2, self.H)
        return hm.hm_combine(self.y, None, self.plan, torch.empty_like(x))

    def backward(self, gout: torch.Tensor, gtotal=None):
        """gout [T, H] bf16 -> gradients of x (bf16), gate, w13 and w2 (fp32), and of the norm's weight if there is one; that
        of x is the residual's too, and gtotal what comes past the layer."""
        plan, empty = self.plan, lambda *shape: torch.empty(shape, dtype=torch.float32, device=gout.device)
        g_weights = hm.hm_combine_weight_grad(gout, self.y, plan, empty(*self.ids.shape))
        g_logits = hm.hm_route_backward(self.logits, self.router, self.ids, g_weights, torch.empty_like(self.logits))
        packed = lambda: torch.zeros((self.rows, self.H), dtype=torch.bfloat16, device=gout.device)
        g_y = hm.hm_combine_transpose_bf16(gout, plan, packed())
        g_a = self._product(self._rows8(g_y), self.q2_t, self.F)
        # the gradient of [gate | up] as rows for theirs and as columns for the weights', and the activation as columns
        _, *g_h = hm.hm_gated_backward(self.h, g_a, plan.dest_offset, None,
                                       *hm.alloc_rows8(self.rows, 2 * self.F, device=gout.device),
                                       *self._alloc_columns8(2 * self.F, gout.device), *self._alloc_columns8(self.F, gout.device))
        g_w2 = hm.hm_expert_matmul_dw(*self._columns8(g_y), *g_h[4:], plan.dest_offset, self.rows,
                                      empty(self.E, self.H, self.F))
        g_rows = self._product(g_h[:2], self.q13_t, self.H)
        rows = hm.hm_dispatch_pack(self.x, plan, packed())
        g_w13 = hm.hm_expert_matmul_dw(*g_h[2:4], *self._columns8(rows), plan.dest_offset, self.rows,
                                       empty(self.E, 2 * self.F, self.H))
        g_x = hm.hm_combine(g_rows, torch.ones_like(self.weights), plan, torch.empty_like(self.x))
        g_x = (g_x.float() + g_logits @ self.gate).to(torch.bfloat16)
        g_gate = g_logits.t() @ self.x.float()
        if self.norm is None:
            return g_x, g_gate, g_w13, g_w2
        g_x, g_norm = hm.hm_rms_norm_backward(g_x, self.normed, self.norm, self.eps, torch.empty_like(self.normed),
                                              empty(self.H), gtotal)
        return g_x, g_gate, g_w13, g_w2, g_norm


def make_layer(E: int, K: int, H: int, F: int, score: str = "softmax", seed: int = 0, norm: bool = False, **how) -> ExpertLayer:
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    r = lambda *shape: torch.randn(shape, generator=g, device="cuda")
    return ExpertLayer(r(E, H) / H ** 0.5, (r(E, 2 * F, H) / H ** 0.5).to(torch.bfloat16),
                       (r(E, H, F) / F ** 0.5).to(torch.bfloat16), hm.Router(E, K, score, **how),
                       norm=1 + 0.1 * r(H) if norm else None)


def main():
    T, E, K, H, F = 4096, 64, 8, 2048, 768
    layer = make_layer(E, K, H, F)
    x, gout = (torch.randn((T, H), device="cuda").to(torch.bfloat16) for _ in range(2))
    for what, n, run in (("forward", T, lambda: layer.forward(x)), ("backward", T, lambda: layer.backward(gout)),
                         ("weights in 8 bits", T, layer.quantize), ("few", 16, lambda: layer.few(x[:16])),
                         ("few", 1, lambda: layer.few(x[:1]))):
        for _ in range(3):
            run()
        torch.cuda.synchronize()
        began = time.perf_counter()
        for _ in range(20):
            run()
        torch.cuda.synchronize()
        ms = (time.perf_counter() - began) / 20 * 1e3
        print("%s of %d tokens, %d of %d experts, %d x %d: %.3f ms" % (what, n, K, E, H, F, ms), flush=True)


if __name__ == "__main__":
    main()
