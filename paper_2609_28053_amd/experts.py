"""Handles of the experts themselves: the router by scores and the gated experts in 8 bits.

``ScoredRouter`` chooses by score plus bias within groups and gives the mixture's weights;
``GatedExperts`` are FFN_e(x) = down_e (g sigmoid(g) u), (g, u) = up_e x, on the rows that
``ExpertRows`` has ordered, with the products in 8-bit codes.  As in ``train``, work is
enqueued on the current stream (or ``stream``) and nothing synchronises.
"""
from __future__ import annotations

import contextlib

import torch

from . import eqb
from .train import ExpertRows, _as_stream, _Handle


class ScoredRouter:
    """Routing by scores (eqb.eqb_route_scored).  score: "sigmoid" or "softmax"; groups, top_groups, group_top, normalize
    and scale as there.  bias [E] binary32 is read by every call, so that a balancer may change it in place between
    two steps."""

    def __init__(self, E: int, K: int, bias=None, score: str = "sigmoid", groups: int = 1, top_groups: int = 1,
                 group_top: int = 1, normalize: bool = True, scale: float = 1.0):
        self.E, self.K, self.bias = E, K, bias
        self.score = {"sigmoid": eqb.EQB_SCORE_SIGMOID, "softmax": eqb.EQB_SCORE_SOFTMAX}[score]
        self.groups, self.top_groups, self.group_top = groups, top_groups, group_top
        self.normalize, self.scale = normalize, scale

    def _on(self, stream, *given):
        if stream is None:
            return contextlib.nullcontext()
        stream = _as_stream(stream)
        for t in given:
            if isinstance(t, torch.Tensor) and t.is_cuda:
                t.record_stream(stream)
        return torch.cuda.stream(stream)

    def forward(self, z, stream=None):
        """topk_idx [T,K] and topk_weight [T,K] of the logits z [T,E]."""
        if z.shape[1] != self.E:
            raise ValueError(f"z has {z.shape[1]} experts, the router {self.E}")
        with self._on(stream, z, self.bias):
            idx = torch.empty((z.shape[0], self.K), dtype=torch.int32, device=z.device)
            weight = torch.empty((z.shape[0], self.K), dtype=torch.float32, device=z.device)
            eqb.eqb_route_scored(z, self.bias, self.K, idx, weight, self.score, self.groups, self.top_groups, self.group_top,
                                 self.normalize, self.scale)
        return idx, weight

    def backward(self, z, topk_idx, grad_weight, grad_z=None, stream=None):
        """The gradient with respect to z [T,E] binary32 (grad_weight: ExpertRows.combine_backward's)."""
        with self._on(stream, z, topk_idx, grad_weight, grad_z):
            if grad_z is None:
                grad_z = torch.empty(z.shape, dtype=torch.float32, device=z.device)
            eqb.eqb_route_scored_backward(z, topk_idx, grad_weight, grad_z, self.score, self.normalize, self.scale)
        return grad_z


class _Weights:
    """One tensor of experts' weights [E,N,H] as codes, both ways."""

    def __init__(self, w):
        E, N, H = w.shape
        up = lambda n: -(-n // eqb.EQB_CODE_BLOCK)  # noqa: E731
        new = lambda dtype, *s: torch.empty(s, dtype=torch.uint8, device=w.device).view(dtype)  # noqa: E731
        self.shape = (E, N, H)
        self.codes, self.codes_t = new(eqb._CODES, E, N, eqb.eqb_code_width(H)), new(eqb._CODES, E, H, eqb.eqb_code_width(N))
        self.scales = new(eqb._SCALES, E, up(N), eqb.eqb_scale_width(H))
        self.scales_t = new(eqb._SCALES, E, up(H), eqb.eqb_scale_width(N))

    def check(self, w):
        if tuple(w.shape) != self.shape:
            raise ValueError(f"weights have shape {tuple(w.shape)}, expected {self.shape}")
        eqb._ptr(w, tuple(eqb._ROW_TYPES), name="weights")

    def take(self, w):
        eqb.eqb_quantize_weights(w, self.codes, self.scales, self.codes_t, self.scales_t)

    def all(self):
        return self.codes, self.scales, self.codes_t, self.scales_t


class GatedExperts(_Handle):
    """Gated experts of up [E,2F,H] and down [E,H,F] on the rows of an ``ExpertRows`` plan.  The weights are laid out as
    codes here and by ``refresh`` (after an optimizer step).  forward(train=False) reads nothing but the codes."""

    def __init__(self, up, down):
        E, F2, H = up.shape
        if F2 % 2 or tuple(down.shape) != (E, H, F2 // 2):
            raise ValueError(f"up {tuple(up.shape)} and down {tuple(down.shape)} are not [E,2F,H] and [E,H,F]")
        self.E, self.F, self.H = E, F2 // 2, H
        self.up, self.down = _Weights(up), _Weights(down)
        self.refresh(up, down)
        self._filled(up.device)

    def _buffers(self):
        return (*self.up.all(), *self.down.all())

    def refresh(self, up, down, stream=None):
        """Takes over new weights; ones that do not fit change nothing."""
        self.up.check(up)
        self.down.check(down)
        with self._on(stream, up, down):
            self.up.take(up)
            self.down.take(down)

    def _width(self, x, name):
        if x.shape[1] != self.H:              # other rows may have as many codes
            raise ValueError(f"{name} has rows of {x.shape[1]} elements, the experts take {self.H}")

    def _codes(self, rows, hidden, device):
        return (torch.empty((rows, eqb.eqb_code_width(hidden)), dtype=torch.uint8, device=device).view(eqb._CODES),
                torch.empty((rows, eqb.eqb_scale_width(hidden)), dtype=torch.uint8, device=device).view(eqb._SCALES))

    def _product(self, codes, weights, transposed, offsets, width, dtype):
        out = torch.empty((codes[0].shape[0], width), dtype=dtype, device=offsets.device)
        eqb.eqb_experts_product(*codes, *(weights.all()[2:] if transposed else weights.all()[:2]), offsets, out)
        return out

    def _columns(self, x, offsets, gated=False):
        codes = self._codes(self.F if gated else x.shape[1], eqb.eqb_column_width(x.shape[0], self.E), x.device)
        (eqb.eqb_gated_quantize_columns if gated else eqb.eqb_quantize_columns)(x, offsets, *codes)
        return codes

    def forward(self, x, rows: ExpertRows, stream=None, train=True, plan=None):
        """What the experts return [T*K,H] (rows past offsets[E] are not written) for the tokens x [T,H], and what backward
        takes of it.  plan: (offsets, slot) of another plan than the newest of `rows`."""
        offsets, slot = (rows.offsets, rows.slot) if plan is None else plan
        if offsets is None:
            raise ValueError("no plan has been made")
        self._width(x, "x")
        with self._on(stream, x, offsets, slot):
            R, count = slot.numel(), offsets[self.E:]
            codes = self._codes(R, self.H, x.device)
            eqb.eqb_dispatch_quantized(x, slot, *codes)
            gate = self._product(codes, self.up, False, offsets, 2 * self.F, x.dtype)
            hidden = self._codes(R, self.F, x.device)
            eqb.eqb_gated_quantize(gate, *hidden, count)
            out = self._product(hidden, self.down, False, offsets, self.H, x.dtype)
        return out, ((x, gate, offsets, slot) if train else None)

    def backward(self, grad_out, saved, stream=None):
        """Gradients with respect to the dispatched rows [T*K,H] (ExpertRows.combine without weights gives the tokens'),
        to up and to down (binary32); grad_out [T*K,H] is the combine's gradient of what forward returned.  In between, the
        gradients of the hidden rows and of the gate are of x's type."""
        x, gate, offsets, slot = saved
        self._width(grad_out, "grad_out")
        with self._on(stream, grad_out, x, gate, offsets, slot):
            R, count = grad_out.shape[0], offsets[self.E:]
            new = lambda *s: torch.empty(s, dtype=torch.float32, device=x.device)  # noqa: E731
            codes = self._codes(R, self.H, x.device)
            eqb.eqb_quantize_rows(grad_out, *codes, count)
            grad_hidden = self._product(codes, self.down, True, offsets, self.F, x.dtype)
            grad_down = new(self.E, self.H, self.F)
            eqb.eqb_experts_grad_weight(*self._columns(grad_out, offsets), *self._columns(gate, offsets, gated=True), offsets, grad_down)
            grad_gate = torch.empty_like(gate)
            eqb.eqb_gated_backward(grad_hidden, gate, grad_gate, count)
            codes = self._codes(R, 2 * self.F, x.device)
            eqb.eqb_quantize_rows(grad_gate, *codes, count)
            grad_rows = self._product(codes, self.up, True, offsets, self.H, x.dtype)
            dispatched = torch.empty((R, self.H), dtype=x.dtype, device=x.device)
            eqb.eqb_dispatch(x, slot, dispatched)
            grad_up = new(self.E, 2 * self.F, self.H)
            eqb.eqb_experts_grad_weight(*self._columns(grad_gate, offsets), *self._columns(dispatched, offsets), offsets, grad_up)
        return grad_rows, grad_up, grad_down
