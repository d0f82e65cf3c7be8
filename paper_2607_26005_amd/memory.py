"""What a policy remembers over the steps of an episode, on the device: a gated linear
recurrence.

The paper's policy decides from the views of one step (Sec. 3.3); a policy that should
know what it saw before carries a state from step to step.  These functions are the
layers of one: in training they run over whole sequences of steps (rollouts, recorded
drives, several of either packed behind one another), when acting one step at a time on
a state that stays on the device.  Every one runs in the library's kernels
(csrc/pictura_memory.hip) on the current stream and never waits for the device.
"""
from __future__ import annotations

from typing import Optional

import torch

from paper_2607_26005_amd import pictura
from paper_2607_26005_amd.pictura import EINVAL, PicturaError


def _steps_first(t: torch.Tensor) -> bool:
    return t.stride(1) > t.stride(0)


def _like(t: torch.Tensor) -> torch.Tensor:
    """An uninitialised [batch, steps, channels] tensor in t's order of batch and steps."""
    B, T, C = t.shape
    if _steps_first(t):
        return torch.empty(T, B, C, dtype=t.dtype, device=t.device).transpose(0, 1)
    return torch.empty(B, T, C, dtype=t.dtype, device=t.device)


def _scan(gates, inputs, state, resets, save):
    B, T, C = inputs.shape
    f32 = dict(dtype=torch.float32, device=inputs.device)
    out, last = _like(inputs), torch.empty(B, C, **f32)
    saved = torch.empty(-(-T // pictura.SCAN_STEPS), B, C, **f32) if save else None
    pictura.pictura_gated_scan(gates, inputs, out, last, saved, state, resets)
    return out, last, saved


class _GatedScan(torch.autograd.Function):
    @staticmethod
    def forward(ctx, gates, inputs, state, resets):
        out, last, saved = _scan(gates.detach(), inputs.detach(), None if state is None else state.detach(), resets, True)
        ctx.save_for_backward(gates, inputs, saved, resets)
        ctx.set_materialize_grads(False)
        return out, last

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dout, dlast):
        gates, inputs, saved, resets = ctx.saved_tensors
        if dout is None:
            dout = torch.zeros(inputs.shape[2], dtype=inputs.dtype, device=inputs.device).expand(inputs.shape)
        elif dout.is_neg() or (dout.shape[2] > 1 and dout.stride(2) != 1):
            dout = dout.resolve_neg().clone(memory_format=torch.contiguous_format)
        if dlast is not None:
            dlast = dlast.resolve_neg().contiguous()
        dgates, dinputs = _like(gates), _like(inputs)
        dstate = torch.empty(saved.shape[1:], dtype=torch.float32, device=saved.device) if ctx.needs_input_grad[2] else None
        pictura.pictura_gated_scan_gradient(gates, inputs, saved, dout, dlast, dgates, dinputs, dstate, resets)
        return dgates, dinputs, dstate, None


def gated_scan(gates: torch.Tensor, inputs: torch.Tensor, state: Optional[torch.Tensor] = None,
               resets: Optional[torch.Tensor] = None):
    """(out [batch, steps, channels], state after the last step float32 [batch, channels]) of
    the recurrence h_t = a_t h_(t-1) + (1 - a_t) inputs_t with a = sigmoid(gates).

    gates and inputs: float32, bfloat16 or float16, any strides of batch and steps (a
    rollout's [steps, batch, channels] transposed is as good), channels contiguous.  The
    recurrence runs in float32; out has the inputs' type.  state: what is remembered before
    the first step (None: nothing).  resets, bool or uint8 [batch, steps]: where true, an
    episode begins with that step, and what came before is forgotten.

    Gradients flow to gates, inputs and state."""
    for name, t in (("gates", gates), ("inputs", inputs), ("state", state)):
        if not isinstance(t, torch.Tensor) and (t is not None or name != "state"):
            raise PicturaError(EINVAL, f"{name}: expected a torch tensor on the HIP device, got {type(t).__name__}")
    if inputs.dim() != 3:
        raise PicturaError(EINVAL, f"inputs: shape {tuple(inputs.shape)}, expected [batch, steps, channels]")
    if torch.is_grad_enabled() and (gates.requires_grad or inputs.requires_grad or (state is not None and state.requires_grad)):
        return _GatedScan.apply(gates, inputs, state, resets)
    return _scan(gates, inputs, state, resets, False)[:2]


def gated_step(gates: torch.Tensor, inputs: torch.Tensor, state: torch.Tensor, resets: Optional[torch.Tensor] = None,
               out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """One step of gated_scan's recurrence for [batch, channels], the policy's form when it
    acts: `state` (float32) is replaced by what is remembered after the step, and returned in
    the inputs' type (in `out`, where that is given; it may be the inputs or the gates).
    resets: [batch].  No gradient flows through it."""
    if out is None:
        if not isinstance(inputs, torch.Tensor):
            raise PicturaError(EINVAL, f"inputs: expected a torch tensor on the HIP device, got {type(inputs).__name__}")
        out = torch.empty(inputs.shape, dtype=inputs.dtype, device=inputs.device)
    pictura.pictura_gated_step(gates, inputs, out, state, resets)
    return out
