"""Buffers and handles for training an MoE layer around its routing.

Each class owns the buffers of one operator and makes the calls of ``eqb`` on
them; all computation happens in the library's kernels.  Work is enqueued on
the current stream (or ``stream``), nothing synchronises.

With ``stream`` the caller orders that stream behind the work that makes the
arguments.  What a call returns is allocated on the stream that it is computed
on; a handle's own buffers, which its constructor fills on the stream current
there, and the arguments stay allocated until the work on ``stream`` is done.
Calls of one handle on several streams are ordered by the caller.
"""
from __future__ import annotations

import contextlib

import torch

from . import eqb


def _as_stream(stream):
    """A torch stream of what ``stream`` may be: one, a handle as a number, or None for the current one."""
    if stream is None:
        return torch.cuda.current_stream()
    if hasattr(stream, "cuda_stream"):
        return stream
    return torch.cuda.ExternalStream(int(stream)) if int(stream) else torch.cuda.default_stream()


class _Handle:
    """A handle's buffers and the streams that are behind their fills."""

    _fill = None

    def _filled(self, device):
        """After the constructor's fills on the current stream."""
        device = torch.device(device)
        if device.type == "cuda":
            stream = torch.cuda.current_stream(device)
            self._fill = torch.cuda.Event()
            self._fill.record(stream)
            self._behind = {stream.cuda_stream}

    def _buffers(self):
        """The handle's own buffers that calls on any stream use."""
        return ()

    def _on(self, stream, *given):
        """The context of a call on a stream: what it allocates is the stream's, and the handle's buffers (at its first
        call there) and the given tensors are known to be used there."""
        if self._fill is None:                # no GPU buffers: the call itself says so
            return contextlib.nullcontext()
        first = eqb._stream(stream) not in self._behind
        if stream is None and not first:
            return contextlib.nullcontext()
        stream = _as_stream(stream)
        if first:
            with torch.cuda.stream(stream):
                capturing = torch.cuda.is_current_stream_capturing()
            if not capturing:                 # a capture begins behind all work, and may wait for none of it
                stream.wait_event(self._fill)
                self._behind.add(stream.cuda_stream)
            for t in self._buffers():
                t.record_stream(stream)
        for t in given:
            if isinstance(t, torch.Tensor) and t.is_cuda:
                t.record_stream(stream)
        return torch.cuda.stream(stream)


class ExpertRows(_Handle):
    """The experts' rows of T tokens (Eq. 1): the order of the routed pairs,
    dispatch of the tokens' rows, combine of what the experts return, and the
    gradients of both.  Expert e's rows are offsets[e] .. offsets[e + 1] - 1.

    A plan writes new ``offsets`` and ``slot``; the calls take the newest
    ``slot`` unless they are given one, so that with several batches in flight
    (gradient accumulation) each keeps its own."""

    def __init__(self, T: int, E: int, K: int, device="cuda"):
        self.T, self.E, self.K = T, E, K
        self.offsets = self.slot = None
        self.workspace = torch.empty(eqb.eqb_dispatch_workspace_size(T, K, E), dtype=torch.uint8,
                                     device=torch.device(device))
        self._filled(device)

    def _buffers(self):
        return (self.workspace,)

    def _slot(self, slot):
        if slot is None and self.slot is None:
            raise ValueError("no plan has been made")
        return self.slot if slot is None else slot

    def plan(self, topk_idx, stream=None):
        """Orders the pairs of topk_idx [T,K]; entries outside [0, E) are dropped."""
        with self._on(stream, topk_idx):
            i32 = dict(dtype=torch.int32, device=self.workspace.device)
            offsets, slot = torch.empty(self.E + 1, **i32), torch.empty((self.T, self.K), **i32)
            eqb.eqb_dispatch_plan(topk_idx, self.E, offsets, slot, self.workspace)
        self.offsets, self.slot = offsets, slot
        return self

    def dispatch(self, x, rows=None, stream=None, slot=None):
        """The tokens' rows x [T,H] in the experts' order [T*K,H] (rows past offsets[E] are not written)."""
        slot = self._slot(slot)
        with self._on(stream, x, rows, slot):
            if rows is None:
                rows = torch.empty((self.T * self.K, x.shape[1]), dtype=x.dtype, device=x.device)
            eqb.eqb_dispatch(x, slot, rows)
        return rows

    def combine(self, rows, weight=None, y=None, stream=None, slot=None):
        """sum_k weight[t, k] rows[slot[t, k]] for every token; without weight, the gradient of dispatch."""
        slot = self._slot(slot)
        with self._on(stream, rows, weight, y, slot):
            if y is None:
                y = torch.empty((self.T, rows.shape[1]), dtype=rows.dtype, device=rows.device)
            eqb.eqb_combine(rows, slot, weight, y)
        return y

    def combine_backward(self, grad_y, rows, weight, grad_rows=None, grad_weight=None, stream=None, slot=None):
        """Gradients of combine with respect to the rows and to the weights (the router backward's grad_score)."""
        slot = self._slot(slot)
        with self._on(stream, grad_y, rows, weight, grad_rows, grad_weight, slot):
            if grad_rows is None:
                grad_rows = torch.empty_like(rows)
            if grad_weight is None:
                grad_weight = torch.empty_like(weight)
            eqb.eqb_combine_backward(grad_y, rows, slot, weight, grad_rows, grad_weight)
        return grad_rows, grad_weight


class BalanceLoss(_Handle):
    """The auxiliary balance loss of P groups over T tokens, its loads, and its
    gradient with the router backward.  score: "sigmoid" (normalised) or
    "softmax".

    Every forward writes new ``load``, ``tokens``, ``prob`` and ``loss``;
    ``saved`` is what its gradient takes of them.  backward takes the newest
    unless it is given one: with several batches in flight (gradient
    accumulation) each keeps its own."""

    def __init__(self, T: int, E: int, K: int, P: int = 1, alpha: float = 1e-2, score: str = "sigmoid", device="cuda"):
        self.T, self.E, self.K, self.P, self.alpha = T, E, K, P, alpha
        self.score = {"sigmoid": eqb.EQB_SCORE_SIGMOID, "softmax": eqb.EQB_SCORE_SOFTMAX}[score]
        dev = torch.device(device)
        self.load = self.tokens = self.prob = self.loss = None
        self.workspace = torch.zeros(eqb.eqb_balance_workspace_size(E, P), dtype=torch.uint8, device=dev)
        self._filled(dev)

    def _buffers(self):
        return (self.workspace,)

    def forward(self, z, topk_idx=None, valid=None, part_off=None, load=None, stream=None):
        """The groups' losses [P] (self.loss); counts topk_idx, or takes a copy of the routing's loads (their buffer may
        be the next routing's before the gradient is computed)."""
        if (topk_idx is None) == (load is None):
            raise ValueError("give topk_idx to count, or the loads that the routing counted")
        with self._on(stream, z, topk_idx, valid, load):
            new = dict(device=self.workspace.device)
            if load is None:
                load = torch.empty((self.P, self.E), dtype=torch.int32, **new)
            else:
                eqb._ptr(load, torch.int32, self.P * self.E, "load")
                load = load.clone()
            tokens = torch.empty(self.P, dtype=torch.int32, **new)
            prob = torch.empty((self.P, self.E), dtype=torch.float32, **new)
            loss = torch.empty(self.P, dtype=torch.float32, **new)
            eqb.eqb_balance_loss(z, topk_idx, self.K, self.alpha, load, tokens, prob, loss, self.workspace, valid, part_off,
                                 self.score)
        self.load, self.tokens, self.prob, self.loss = load, tokens, prob, loss
        return loss

    @property
    def saved(self):
        """What the gradient takes of the newest forward."""
        return self.load, self.tokens

    def backward(self, z, grad_loss, grad_z=None, topk_idx=None, grad_score=None, inj=None, valid=None,
                 part_off=None, stream=None, saved=None):
        """The gradient with respect to z; with topk_idx and grad_score (and inj), the whole router's."""
        load, tokens = self.saved if saved is None else saved
        if load is None:
            raise ValueError("no forward has been made")
        with self._on(stream, z, grad_loss, grad_z, topk_idx, grad_score, inj, valid, load, tokens):
            if grad_z is None:
                grad_z = torch.empty((self.T, self.E), dtype=torch.float32, device=z.device)
            eqb.eqb_balance_backward(z, load, tokens, self.K, self.alpha, grad_loss, grad_z, topk_idx, grad_score, inj, valid,
                                     part_off, self.score)
        return grad_z


class AdamW(_Handle):
    """AdamW over a list of binary32 parameters, in place, one call a step.
    state_bits: 32, or 8 for E4M3 states with a scale per 256 elements.
    copies: BF16 tensors that receive the new parameters.  weight_decay: one
    value, or one per parameter.  Every step takes the memory that parameters,
    copies and states have then, and lr, betas, eps, weight_decay and seed as
    they are then.  device_steps: the number of steps taken is kept on the
    device from the start, as steps that are captured in a graph need; else it
    moves there with the first found_inf, which may skip steps without the host
    knowing.  Reading ``steps`` then waits for the current stream, and
    load_state_dict copies there."""

    def __init__(self, params, lr=1e-3, betas=(0.9, 0.95), eps=1e-8, weight_decay=0.0, state_bits=32, copies=None,
                 seed=0, device_steps=False):
        if state_bits not in (8, 32):
            raise ValueError(f"state_bits is 8 or 32, not {state_bits}")
        self.params, self.lr, self.betas, self.eps, self.seed = list(params), lr, betas, eps, seed
        self._counter, self.steps = None, 0
        self.weight_decay, self.copies, self.state_bits = weight_decay, copies, state_bits
        if state_bits == 8:
            new = lambda: [torch.zeros(p.shape, dtype=torch.uint8, device=p.device).view(torch.float8_e4m3fn)  # noqa: E731
                           for p in self.params]
            scales = lambda: [torch.zeros(-(-p.numel() // eqb.EQB_ADAMW_BLOCK), device=p.device)  # noqa: E731
                              for p in self.params]
            self.exp_avg_scale, self.exp_avg_sq_scale = scales(), scales()
        else:
            new = lambda: [torch.zeros_like(p) for p in self.params]  # noqa: E731
            self.exp_avg_scale = self.exp_avg_sq_scale = None
        self.exp_avg, self.exp_avg_sq = new(), new()
        self._tensors = None
        if device_steps and self.params:
            self._count_on_device()
        self._filled(self.params[0].device if self.params else "cpu")

    def _buffers(self):
        return [t for ts in (self.params, self.copies, self.exp_avg, self.exp_avg_sq, self.exp_avg_scale,
                             self.exp_avg_sq_scale, None if self._counter is None else [self._counter]) for t in ts or ()]

    @property
    def steps(self) -> int:
        """The steps taken: those that found_inf skipped are none."""
        return self._steps if self._counter is None else int(self._counter[0])

    @steps.setter
    def steps(self, n):
        if self._counter is None:
            self._steps = int(n)
        else:
            self._counter[0].fill_(int(n))

    def _count_on_device(self):
        counter = torch.zeros(eqb.EQB_ADAMW_COUNTER_BYTES // 8, dtype=torch.int64, device=self.params[0].device)
        counter[0].fill_(self._steps)
        self._counter = counter

    def step(self, grads, lr=None, grad_scale=None, found_inf=None, stream=None):
        """One step with these gradients, one per parameter, all binary32 or all BF16.  Where the device scalar
        found_inf is not 0 nothing changes, the number of steps included."""
        tensors = (self.params, self.exp_avg, self.exp_avg_sq, self.copies, self.exp_avg_scale, self.exp_avg_sq_scale,
                   self.weight_decay)
        if self._tensors is None:
            self._tensors = eqb.AdamwTensors(self.params, grads, *tensors[1:])
        else:
            if self._tensors.refresh(*tensors) and self._fill is not None:
                self._behind.clear()          # memory that no stream is known to use
            self._tensors.set_grads(grads)
        with self._on(stream, grad_scale, found_inf, *grads):
            if self._counter is None and torch.cuda.is_initialized() and torch.cuda.is_current_stream_capturing():
                raise RuntimeError("a captured step needs AdamW(device_steps=True): replays would repeat one step's number")
            if self._counter is None and found_inf is not None and self.params:
                self._count_on_device()
                self._behind.clear()
            numbers = (self.lr if lr is None else lr, *self.betas, self.eps, self.seed, grad_scale, found_inf)
            if self._counter is None:
                eqb.eqb_adamw_step(self._tensors, self._steps + 1, *numbers)
                self._steps += 1
            else:
                eqb.eqb_adamw_step_counted(self._tensors, self._counter, *numbers)
        # autograd sees that what it kept of them for a backward pass has changed
        torch.autograd.graph.increment_version([*self.params, *(self.copies or ())])

    def state_dict(self) -> dict:
        """The number of steps taken and the states (the optimizer's own tensors, not copies)."""
        return dict(steps=self.steps, exp_avg=self.exp_avg, exp_avg_sq=self.exp_avg_sq,
                    exp_avg_scale=self.exp_avg_scale, exp_avg_sq_scale=self.exp_avg_sq_scale)

    def load_state_dict(self, state: dict) -> None:
        """Takes over the values of a state_dict of the same parameters and state_bits; one that does not fit changes
        nothing."""
        names = ("exp_avg", "exp_avg_sq", "exp_avg_scale", "exp_avg_sq_scale")
        steps = int(state["steps"])
        for name in names:
            mine, theirs = getattr(self, name), state[name]
            if (mine is None) != (theirs is None):
                raise ValueError(f"the state is not one of {self.state_bits} bits")
            if mine is None:
                continue
            fits = [t.shape == u.shape and (t.dtype is u.dtype or (t.dtype is torch.float32 and u.is_floating_point()))
                    for t, u in zip(mine, theirs)]
            if len(mine) != len(theirs) or not all(fits):
                raise ValueError(f"{name} has other shapes or types")
        for name in names:
            for a, b in zip(getattr(self, name) or (), state[name] or ()):
                a.copy_(b)
        self.steps = steps
