"""The policy's decisions and its training step, on the device: actions drawn from
the head's logits, the clipped policy loss and a preference loss over pairs of sequences
with their gradients, and AdamW.

The paper trains its perspective policy in the process that renders for it
(Sec. 3.3; App. A.3, table of hyperparameters: clipped policy optimisation with
clip 0.2 and normalised advantages, AdamW).  `encoder.ViewEncoder` turns rendered
views into a scene embedding; these functions are what acts and learns behind it.
Every one runs in the library's kernels (csrc/pictura_policy.hip,
csrc/pictura_prefer.hip, csrc/pictura_adamw.hip) on the current stream and never waits for the device.
"""
from __future__ import annotations

import operator
from typing import NamedTuple, Optional

import numpy as np
import torch
from torch.optim import optimizer as _optimizer

from paper_2607_26005_amd import _tensors, pictura
from paper_2607_26005_amd.pictura import EINVAL, PicturaError

pictura._bind_helper(_tensors)

POLICY_STATS = pictura.POLICY_STATS
PREFERENCE_STATS = pictura.PREFERENCE_STATS


def sample_actions(logits: torch.Tensor, uniform: torch.Tensor, mask: Optional[torch.Tensor] = None, temperature=1.0,
                   top_k=0, top_p=1.0, min_p=0.0):
    """(actions int64 [rows], log-probabilities float32 [rows]) drawn from logits
    [rows, actions] by the numbers uniform [rows] in [0, 1): the same logits and
    numbers give the same actions, whatever else is in the batch.

    mask (bool or uint8, [rows, actions] or [actions]): 0 where an action is not
    allowed.  temperature (0: the largest logit; infinity: all allowed actions of
    finite logit alike), top_k, top_p and min_p are numbers or tensors of one per row
    (float32; top_k int32); 0, 1 and 0 turn the filters off.  A row without an allowed
    action, or with a NaN, gives -1 and NaN.  The log-probability is that of the
    distribution drawn from, after temperature and filters.  No gradient flows
    through a draw."""
    N = logits.shape[0] if isinstance(logits, torch.Tensor) and logits.dim() == 2 else 0
    dev = logits.device if isinstance(logits, torch.Tensor) else None
    actions = torch.empty(N, dtype=torch.int64, device=dev)
    logp = torch.empty(N, dtype=torch.float32, device=dev)
    pictura.pictura_sample_actions(logits, uniform, actions, logp, mask, temperature, top_k, top_p, min_p)
    return actions, logp


class PolicyGradient(NamedTuple):
    stats: torch.Tensor     # float32 [6], see POLICY_STATS
    dlogits: torch.Tensor   # the logits' type and shape
    dvalues: torch.Tensor   # float32 [rows]


def policy_gradient(logits, values, actions, old_logp, advantages, returns, *, old_values=None, weights=None, mask=None,
                    temperature: float = 1.0, clip: float = 0.2, value_clip: float = 0.0, value_coef: float = 0.5,
                    entropy_coef: float = 0.01, normalize: bool = False, denominator: float = 0.0) -> PolicyGradient:
    """The clipped policy loss over a batch of decisions and its gradient with respect
    to logits and values, in one pass over the logits (the formulas stand at
    pictura_policy_loss in include/pictura.h).

    weights [rows]: rows of weight 0 count nothing (an advantage filter), nor do rows
    whose action is outside the head (-1 from sample_actions).  The loss is the mean
    by weight, or the sum over `denominator` where that is given: parts of a
    minibatch then add up.  normalize: advantages by the mean and deviation of the
    rows given here.  value_clip > 0 needs old_values.

    dlogits is cut to the logits' type here, before any factor of the caller's: in float16,
    entries below 2^-24 are lost.  policy_loss keeps them; so does a denominator that
    is smaller by the loss scale, with dlogits and dvalues that much larger."""
    if not isinstance(logits, torch.Tensor):
        raise PicturaError(EINVAL, f"logits: expected a torch tensor on the HIP device, got {type(logits).__name__}")
    stats = torch.empty(len(POLICY_STATS), dtype=torch.float32, device=logits.device)
    dlogits = torch.empty(logits.shape, dtype=logits.dtype, device=logits.device)
    dvalues = torch.empty(logits.shape[:1], dtype=torch.float32, device=logits.device)
    pictura.pictura_policy_loss(logits, values, actions, old_logp, advantages, returns, stats, dlogits, dvalues,
                                old_values, weights, mask, temperature, clip, value_clip, value_coef, entropy_coef,
                                normalize, denominator)
    return PolicyGradient(stats, dlogits, dvalues)


class _PolicyLoss(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, values, args, kwargs):
        # float16's range is too short for a gradient that a loss scale has yet to lift (of
        # 65,536 rows of 12 a third of the entries would be 0): kept in float32 until then
        x = logits.detach()
        out = policy_gradient(x.float() if x.dtype == torch.float16 else x, values.detach(), *args, **kwargs)
        ctx.dtype = x.dtype
        ctx.save_for_backward(out.dlogits, out.dvalues)
        ctx.mark_non_differentiable(out.stats)
        return out.stats[0].clone(), out.stats

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dloss, _):
        dlogits, dvalues = ctx.saved_tensors
        # (the product in fp32: a loss scale may be beyond what the logits' type holds)
        if ctx.dtype == torch.float32:
            dx = dlogits * dloss
        else:
            dx = torch.empty(dlogits.shape, dtype=ctx.dtype, device=dlogits.device)
            torch.mul(dlogits.float(), dloss, out=dx)
        return dx, dvalues * dloss, None, None


def policy_loss(logits, values, actions, old_logp, advantages, returns, **kwargs):
    """(loss, stats) for autograd: policy_gradient's loss, whose backward hands on the
    gradient that the same pass computed, times the factor that arrives (a loss scale).
    Only logits and values get one.  Of float16 logits the gradient is kept in float32
    for that, 4 bytes an entry (and 4 more for the logits' copy while it is computed)."""
    return _PolicyLoss.apply(logits, values, (actions, old_logp, advantages, returns), kwargs)


class PreferenceGradient(NamedTuple):
    stats: torch.Tensor     # float32 [4], see PREFERENCE_STATS
    dlogits: torch.Tensor   # the logits' type and shape
    ratios: torch.Tensor    # float32 [2 pairs], the sequences' log ratios


def preference_gradient(logits, actions, offsets, ref_logp=None, *, weights=None, mask=None, beta: float = 0.1,
                        smoothing: float = 0.0, average: bool = False, denominator: float = 0.0) -> PreferenceGradient:
    """The preference loss over pairs of sequences of decisions and its gradient with
    respect to the logits (the formulas stand at pictura_preference_loss in
    include/pictura.h).

    Row n of logits is a decision whose action was actions[n]; sequence s is the rows from
    offsets[s] on up to offsets[s + 1] (int64 [2 pairs + 1], on the device), and of pair p
    sequence 2p is the one preferred to sequence 2p + 1.  ref_logp [rows]: the actions'
    log-probabilities by the policy that is not to be left too far (None: 0).  Padded
    sequences are ones whose further rows have action -1.  Sequences are best of like lengths:
    with heads of up to 64 actions one pair far longer than the others is a workgroup's alone.

    weights [pairs]; the loss is the mean by weight, or the sum over `denominator` where that
    is given: parts of a minibatch then add up.  average: a sequence's log ratio is the mean
    over its rows in place of the sum.  smoothing: labels are wrong that often.

    dlogits is cut to the logits' type here, before any factor of the caller's; preference_loss
    keeps what float16 would lose.  Both are refused where they would not be seen: under
    torch.jit.trace, torch.func's transforms and dispatch modes, and for tensors with a tangent."""
    try:
        return PreferenceGradient(*_tensors.preference_gradient(logits, actions, offsets, ref_logp, weights, mask, beta,
                                                                smoothing, average, denominator))
    except ValueError as e:
        raise PicturaError(EINVAL, str(e)) from None


def preference_loss(logits, actions, offsets, ref_logp=None, *, weights=None, mask=None, beta: float = 0.1,
                    smoothing: float = 0.0, average: bool = False, denominator: float = 0.0):
    """(loss, stats, ratios) for autograd: preference_gradient's loss, whose backward hands
    on the gradient that the same call computed, times the factor that arrives (a loss
    scale).  Only the logits get one: a ref_logp or weights that want a gradient are refused.
    Of float16 logits the gradient is kept in float32 for that; of bfloat16 ones in bfloat16, so
    that a factor rounds it once more."""
    try:
        return _tensors.preference_loss(logits, actions, offsets, ref_logp, weights, mask, beta, smoothing, average,
                                        denominator)
    except ValueError as e:
        raise PicturaError(EINVAL, str(e)) from None


class AdamW(torch.optim.Optimizer):
    """AdamW over all weights in a few launches, with the gradients clipped to a
    common norm (max_norm) and the moments in fp32 (bits=32) or in 8 bits with a
    scale for each 256 elements (bits=8: 2.03 bytes of state a weight in place of 8).

    Weights and gradients: float32, bfloat16 or float16, contiguous, on one device.
    step(grads=...) takes the gradients as a list in the order of the parameters
    (None: no gradient) in place of the parameters' own .grad; they may be of another
    type than the weights.  After a step with max_norm, grad_norm is the norm before
    clipping, a tensor on the device.  With bits=8 a weight's state holds codes
    (exp_avg int8, exp_avg_sq uint8) and scales; moments() gives what they stand for.

    The step number is the host's: a step captured in a graph replays with the rate and
    the bias correction that it was captured with, and counts once."""

    def __init__(self, params, lr: float = 1e-3, betas=(0.9, 0.999), eps: float = 1e-8, weight_decay: float = 1e-2,
                 bits: int = 32, max_norm: Optional[float] = None):
        if bits not in (32, 8):
            raise PicturaError(EINVAL, f"bits: {bits}, expected 32 or 8")
        if max_norm is not None and not max_norm >= 0:
            raise PicturaError(EINVAL, f"max_norm: {max_norm}")
        self.bits, self.max_norm = bits, max_norm
        self.grad_norm = None
        super().__init__(params, dict(lr=lr, betas=betas, eps=eps, weight_decay=weight_decay))

    def __getstate__(self):
        # (what torch's own keeps of an optimizer in copies and pickles, and what this one adds)
        return dict(super().__getstate__(), bits=self.bits, max_norm=self.max_norm, grad_norm=self.grad_norm)

    def _state(self, p):
        s = self.state[p]
        if "step" not in s:
            flat = lambda dt, n: torch.zeros(n, dtype=dt, device=p.device)
            n = p.numel()
            s["step"] = 0
            if self.bits == 32:
                s["exp_avg"], s["exp_avg_sq"] = flat(torch.float32, n), flat(torch.float32, n)
            else:
                blocks = -(-n // pictura.ADAMW_BLOCK)
                s["exp_avg"], s["exp_avg_sq"] = flat(torch.int8, n), flat(torch.uint8, n)
                s["exp_avg_scale"], s["exp_avg_sq_scale"] = flat(torch.float32, blocks), flat(torch.float32, blocks)
        return s

    def _in_order(self, params):
        """Whether the states are those of these parameters, one by one (a lookup by
        tensor costs ten times this)."""
        return len(self.state) == len(params) and all(map(operator.is_, self.state, params))

    def _table(self, params, grads):
        """(rows of pictura_adamw_tensor, their steps, the states, the device of all rows) of
        the parameters that have a gradient (grads: a list, or True for the parameters' own;
        False: of all that have a state), everything checked that the kernels rely on."""
        table, steps = np.empty(len(params), pictura.ADAMW_TENSOR), np.empty(len(params), np.int64)
        try:
            states = list(self.state.values()) if self._in_order(params) else None
            got = _tensors.fill(params, grads, states, self.bits, table, steps) if states is not None else None
            if got is None:   # (states that have not begun may be there, empty: to read one makes it)
                if grads is False:
                    states = [self.state[p] for p in params]
                else:
                    states = [self._state(p) if (p.grad if grads is True else g) is not None else None
                              for p, g in zip(params, params if grads is True else grads)]
                got = _tensors.fill(params, grads, states, self.bits, table, steps)
            n, first = got
        except ValueError as e:
            raise PicturaError(EINVAL, str(e)) from None
        if not n:
            return table[:0], steps[:0], states, None
        if not params[first].is_cuda:   # (the first that takes part: those without a gradient may be anywhere)
            pictura._check_device(params[first], f"parameter {first}", None)
        return table[:n], steps[:n], states, params[first].device

    def step(self, closure=None, grads=None):
        if (self._optimizer_step_pre_hooks or self._optimizer_step_post_hooks or _optimizer._global_optimizer_pre_hooks
                or _optimizer._global_optimizer_post_hooks or torch.autograd._profiler_enabled()):
            return self._hooked_step(closure, grads=grads)
        return self._step(closure, grads)

    step.hooked = True   # by _hooked_step: torch's wrapper takes 10 us also where there is nothing to call

    def _step(self, closure=None, grads=None):
        loss = None
        if closure is not None:
            with torch.enable_grad():
                loss = closure()
        params = [p for group in self.param_groups for p in group["params"]]
        if grads is not None and len(grads) != len(params):
            raise PicturaError(EINVAL, f"grads: {len(grads)} of them for {len(params)} parameters")
        table, steps, states, dev = self._table(params, True if grads is None else list(grads))
        if dev is None:
            return loss
        factor = None
        if self.max_norm is not None:
            norm = torch.empty(2, dtype=torch.float32, device=dev)
            pictura.pictura_grad_norm(table, self.max_norm, norm, dev)
            self.grad_norm, factor = norm[0], norm[1:]
        # one call for neighbours of a group at the same step
        got = range(len(params)) if len(table) == len(params) else \
            [i for i, p in enumerate(params) if (p.grad if grads is None else grads[i]) is not None]
        ends, at = [], 0
        for group in self.param_groups:
            at += len(group["params"])
            ends.append(sum(1 for i in got if i < at) if len(table) != len(params) else at)
        begin = 0
        for group, end in zip(self.param_groups, ends):
            while begin < end:
                same = steps[begin:end] != steps[begin]
                stop = begin + int(same.argmax()) if same.any() else end
                pictura.pictura_adamw_step(table[begin:stop], dev, group["lr"], group["betas"], group["eps"],
                                           group["weight_decay"], int(steps[begin]) + 1, self.bits, factor)
                for i in got[begin:stop]:   # (also where a later call is refused: these have moved)
                    states[i]["step"] += 1
                begin = stop
        return loss

    _hooked_step = torch.optim.Optimizer.profile_hook_step(_step)

    @torch.no_grad()
    def moments(self, out=None):
        """(first moments, second moments) of all parameters that have a state, two
        lists of float32 tensors; with bits=8 what the codes stand for, written to
        the two lists of contiguous float32 tensors `out` where that is given."""
        params = [p for group in self.param_groups for p in group["params"]]
        if not self._in_order(params) or not all(["step" in s for s in self.state.values()]):
            params = [p for p in params if "step" in self.state.get(p, ())]
        if self.bits == 32:
            return [self.state[p]["exp_avg"] for p in params], [self.state[p]["exp_avg_sq"] for p in params]
        table, _, _, dev = self._table(params, False)
        if out is None:
            out = tuple([torch.empty(p.numel(), dtype=torch.float32, device=p.device) for p in params] for _ in range(2))
        try:
            addresses = [_tensors.outputs(list(ts), params) for ts in out]
        except ValueError as e:
            raise PicturaError(EINVAL, str(e)) from None
        if dev is not None:
            pictura.pictura_adamw_moments(table, *(np.frombuffer(a, np.uint64) for a in addresses), dev)
        return list(out[0]), list(out[1])

    def state_dict(self):
        """As torch's, with max_norm beside the groups."""
        held = super().state_dict()
        held["max_norm"] = self.max_norm
        return held

    def load_state_dict(self, state_dict):
        """As torch's, with the moments' own types kept (torch would make them the
        weights'), and with max_norm, as the rates of the groups, taken from the
        dictionary where that has it."""
        made = []   # what the hooks before this one make of it; the hooks after see the result
        hooks = (self.register_load_state_dict_pre_hook(lambda _, held: made.append(held)),
                 self.register_load_state_dict_post_hook(lambda _: self._take(made[0]), prepend=True))
        try:
            super().load_state_dict(state_dict)
        finally:
            for hook in hooks:
                hook.remove()

    def _take(self, state_dict):
        self.max_norm = state_dict.get("max_norm", self.max_norm)
        at = {}
        for mine, theirs in zip(self.param_groups, state_dict["param_groups"]):
            at.update(zip(theirs["params"], mine["params"]))
        for key, held in state_dict["state"].items():
            p = at.get(key)
            if p is not None:
                self.state[p] = {k: v.to(device=p.device, copy=True).contiguous() if isinstance(v, torch.Tensor) and k != "step"
                                 else int(v) if k == "step" else v for k, v in held.items()}
