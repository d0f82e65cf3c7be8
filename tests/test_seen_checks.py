"""The calls of memory and of the preference loss are no operators of torch: where what they
compute would be lost without a word (tangents, recorded or transformed programs) they are
refused, before any device work (host tensors; no GPU needed)."""
import pytest
import torch
import torch.autograd.forward_ad as forward_ad
from torch.utils._python_dispatch import TorchDispatchMode

from paper_2607_26005_amd import memory, pictura, policy

z = torch.zeros
N, A = 4, 3
CALLS = {
    "gated_scan": (memory.gated_scan, dict(gates=z(2, 5, 6), inputs=z(2, 5, 6), state=z(2, 6))),
    "gated_step": (memory.gated_step, dict(gates=z(2, 6), inputs=z(2, 6), state=z(2, 6), out=z(2, 6))),
    "rms_norm": (memory.rms_norm, dict(x=z(N, 6), weight=z(6), residual=z(N, 6))),
    "rms_norm_8bit": (memory.rms_norm_8bit, dict(x=z(N, 6), weight=z(6), residual=z(N, 6))),
    "row_values": (lambda scales, out: memory.RowCodes(z(N, 6, dtype=torch.int8), scales, None).values(out),
                   dict(scales=z(N), out=z(N, 6))),
    **{name: (getattr(policy, name), dict(logits=z(N, A), actions=z(N, dtype=torch.int64), offsets=torch.tensor([0, 2, 4]),
                                          ref_logp=z(N), weights=z(1))) for name in ("preference_gradient", "preference_loss")},
}
EACH = [(name, k) for name, (_, a) in CALLS.items() for k, v in a.items() if v.is_floating_point()]


def _raises(match, f, *a, **k):
    with pytest.raises(pictura.PicturaError, match=match) as e:
        f(*a, **k)
    assert e.value.status == pictura.EINVAL


@pytest.mark.parametrize("name, argument", EACH)
def test_a_tangent_is_not_lost(name, argument):
    f, a = CALLS[name]
    with forward_ad.dual_level():
        dual = forward_ad.make_dual(a[argument].clone(), torch.ones_like(a[argument]))
        assert not dual.requires_grad   # (so that asking for a gradient alone does not find it)
        for mode in (torch.enable_grad, torch.no_grad):
            with mode():
                _raises(f"{argument}: has a tangent", f, **dict(a, **{argument: dual}))
        with forward_ad._set_fwd_grad_enabled(False):   # the next check
            _raises("expected the HIP device", f, **dict(a, **{argument: dual}))


@pytest.mark.parametrize("name", CALLS)
def test_a_dispatch_mode_would_not_see_the_call(name):
    class Mode(TorchDispatchMode):
        def __torch_dispatch__(self, func, types, args=(), kwargs=None):
            return func(*args, **(kwargs or {}))

    f, a = CALLS[name]
    with Mode():
        _raises(f"{name}: called under a dispatch mode", f, **a)
    _raises("expected the HIP device", f, **a)


@pytest.mark.parametrize("name", CALLS)
def test_a_transform_would_not_see_the_call(name):
    f, a = CALLS[name]

    def inside(x):
        _raises(f"{name}: called under torch.func", f, **a)
        return x * 2

    torch.func.vmap(inside)(z(3))
    torch.func.grad(inside)(z(()))


@pytest.mark.parametrize("name", CALLS)
def test_a_trace_would_not_see_the_call(name):
    f, a = CALLS[name]

    def inside(x):
        _raises(f"{name}: called under torch.jit.trace", f, **a)
        return x * 2

    torch.jit.trace(inside, z(3), check_trace=False)
