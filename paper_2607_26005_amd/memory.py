"""What a policy remembers over the steps of an episode, on the device: a gated linear
recurrence, and the root-mean-square norm between its layers.

The paper's policy decides from the views of one step (Sec. 3.3); a policy that should
know what it saw before carries a state from step to step.  These functions are the
layers of one: in training they run over whole sequences of steps (rollouts, recorded
drives, several of either packed behind one another), when acting one step at a time on
a state that stays on the device.  Every one runs in the library's kernels
(csrc/pictura_memory.hip, csrc/pictura_norm.hip) on the current stream and never waits for the device.

They are no operators of torch.  What would not see them, and so lose what they compute,
is refused: torch.jit.trace, torch.func's transforms, dispatch modes, and tensors with a
tangent (forward-mode differentiation).
"""
from __future__ import annotations

from typing import NamedTuple, Optional

import torch
import torch.nn as nn

from paper_2607_26005_amd import _tensors, pictura
from paper_2607_26005_amd.pictura import EINVAL, PicturaError

pictura._bind_helper(_tensors)


def gated_scan(gates: torch.Tensor, inputs: torch.Tensor, state: Optional[torch.Tensor] = None,
               resets: Optional[torch.Tensor] = None):
    """(out [batch, steps, channels], state after the last step float32 [batch, channels]) of
    the recurrence h_t = a_t h_(t-1) + (1 - a_t) inputs_t with a = sigmoid(gates).

    gates and inputs: float32, bfloat16 or float16, any strides of batch and steps (a
    rollout's [steps, batch, channels] transposed is as good), channels contiguous.  The
    recurrence runs in float32; out has the inputs' type.  state: what is remembered before
    the first step (None: nothing).  resets, bool or uint8 [batch, steps]: where true, an
    episode begins with that step, and what came before is forgotten.  Sequences packed one
    behind the other are one with resets; padding behind a sequence changes nothing before
    it (with a reset where it begins also if it holds no numbers), but is in the last state.

    Gradients flow to gates, inputs and state."""
    try:
        return _tensors.gated_scan(gates, inputs, state, resets)
    except ValueError as e:
        raise PicturaError(EINVAL, str(e)) from None


def gated_step(gates: torch.Tensor, inputs: torch.Tensor, state: torch.Tensor, resets: Optional[torch.Tensor] = None,
               out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """One step of gated_scan's recurrence for [batch, channels], the policy's form when it
    acts: `state` (float32) is replaced by what is remembered after the step, and returned in
    the inputs' type (in `out`, where that is given; it may be the inputs or the gates, and is
    refused where it overlaps them, the state or the resets in another way).
    resets: [batch].  No gradient flows through it: where one is wanted it is refused."""
    try:
        return _tensors.gated_step(gates, inputs, state, resets, out)
    except ValueError as e:
        raise PicturaError(EINVAL, str(e)) from None


def rms_norm(x: torch.Tensor, weight: torch.Tensor, residual: Optional[torch.Tensor] = None, eps: float = 1e-6):
    """y = s / sqrt(mean(s^2) + eps) * weight over the last dimension of s = x + residual.
    Returns y, or with a residual (y, s): s, rounded to the type, is the residual that goes on.

    x and residual: float32, bfloat16 or float16, rows of 1 to 65,536 (tensors whose rows do
    not stand at one distance are copied first); weight of that type or float32.  The mean is
    taken in 64 bits, the rest in float32.  Gradients flow to x, residual and weight."""
    try:
        return _tensors.rms_norm(x, weight, residual, eps)
    except ValueError as e:
        raise PicturaError(EINVAL, str(e)) from None


class RowCodes(NamedTuple):
    """Rows in 8 bits: what a code stands for is its value times the scale of its row."""
    codes: torch.Tensor            # int8 or float8_e4m3fn, the input's shape
    scales: torch.Tensor           # float32 [...], one for each row
    sum: Optional[torch.Tensor]    # x + residual, where there is a residual

    def values(self, out: Optional[torch.Tensor] = None) -> torch.Tensor:
        """What the codes stand for, float32 (in `out`, contiguous, where that is given).  Has
        no gradient, as the codes."""
        try:
            return _tensors.row_values(self.codes, self.scales, out)
        except ValueError as e:
            raise PicturaError(EINVAL, str(e)) from None


def rms_norm_8bit(x: torch.Tensor, weight: torch.Tensor, residual: Optional[torch.Tensor] = None, eps: float = 1e-6,
                  dtype: torch.dtype = torch.float8_e4m3fn) -> RowCodes:
    """rms_norm with an output in 8 bits, for layers that multiply in them: codes of `dtype`
    (float8_e4m3fn or int8) and a scale for each row, its largest magnitude M over 448 or 127.
    A code is the nearest one of the float32 result y times 448 (1 / M) or 127 (1 / M), each
    operation rounded to float32.  Codes and scales have no
    gradient: where one is wanted it raises when it would reach them (detach them to go
    without).  `sum` hands on its own, to x and the residual."""
    if dtype not in (torch.int8, torch.float8_e4m3fn):
        raise PicturaError(EINVAL, f"dtype: {dtype}, expected float8_e4m3fn or int8")
    try:
        return RowCodes(*_tensors.rms_norm_8bit(x, weight, residual, eps, dtype is not torch.int8))
    except ValueError as e:
        raise PicturaError(EINVAL, str(e)) from None


class MemoryLayer(nn.Module):
    """A layer of a policy that remembers: norm, one projection to gates and inputs, the gated
    recurrence, and a projection back, beside the residual stream.

    x is what the layer before put out and `residual` the stream before that was added (None
    for the first layer): their sum is taken by the norm."""

    def __init__(self, width: int, eps: float = 1e-6):
        super().__init__()
        self.width, self.eps = width, eps
        self.norm = nn.Parameter(torch.ones(width))
        self.project = nn.Linear(width, 2 * width)
        self.out = nn.Linear(width, width)
        with torch.no_grad():   # gates that keep for some ten steps
            self.project.bias[:width] = 2.0

    def _normed(self, x, residual):
        """(what is projected, the stream): the norm, and x as the stream goes on."""
        if residual is None:
            return rms_norm(x, self.norm, None, self.eps), x
        # (under autocast the layer before puts out its products' type, and the stream keeps its own)
        return rms_norm(x.to(residual.dtype), self.norm, residual, self.eps)

    def forward(self, x: torch.Tensor, residual: Optional[torch.Tensor] = None, state: Optional[torch.Tensor] = None,
                resets: Optional[torch.Tensor] = None):
        """x [batch, steps, width] -> (output, residual stream, state after the last step)."""
        y, stream = self._normed(x, residual)
        gates, inputs = self.project(y).chunk(2, -1)
        h, state = gated_scan(gates, inputs, state, resets)
        return self.out(h), stream, state

    def quantized(self):
        """The projection's weights in 8 bits, for `step`: (codes [2 width, width], scales)."""
        w = self.project.weight.detach().float()   # (1e-30 is 0 in float16)
        scales = w.abs().amax(1, keepdim=True).clamp(min=1e-30) / 448.0
        return (w / scales).to(torch.float8_e4m3fn), scales.t().contiguous()

    @torch.no_grad()
    def step(self, x: torch.Tensor, residual: Optional[torch.Tensor], state: torch.Tensor,
             resets: Optional[torch.Tensor] = None, codes=None):
        """One step of [batch, width] on `state` (float32, replaced) -> (output, residual
        stream).  codes (of `quantized`): the projection multiplies in 8 bits (width a multiple
        of 16)."""
        if codes is None:
            y, stream = self._normed(x, residual)
            both = self.project(y)
        else:
            x = x if residual is None else x.to(residual.dtype)
            held = rms_norm_8bit(x, self.norm, residual, self.eps)
            stream = x if residual is None else held.sum
            both = torch._scaled_mm(held.codes, codes[0].t(), scale_a=held.scales[:, None], scale_b=codes[1],
                                    out_dtype=torch.bfloat16).to(x.dtype) + self.project.bias
        gates, inputs = both.chunk(2, -1)
        return self.out(gated_step(gates, inputs, state, resets)), stream
