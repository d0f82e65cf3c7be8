"""The preference loss refuses what its kernels could not use safely, before any device
work: host tensors stand in for device ones (no GPU needed)."""
import ctypes

import pytest
import torch

from paper_2607_26005_amd import pictura, policy

N, A, P = 6, 12, 2
z = torch.zeros


@pytest.fixture(autouse=True)
def host_is_device(request, monkeypatch):
    if "device" not in request.node.name:
        monkeypatch.setattr(pictura, "_check_device", lambda t, name, ctx: None)


def _raises(match, fn, *a, **k):
    with pytest.raises(pictura.PicturaError, match=match) as e:
        fn(*a, **k)
    assert e.value.status == pictura.EINVAL


def _args(**over):
    return dict(dict(logits=z(N, A), actions=z(N, dtype=torch.int64), offsets=z(2 * P + 1, dtype=torch.int64), ref_logp=z(N)), **over)


@pytest.mark.parametrize("match, bad", [
    ("logits: expected a torch tensor", dict(logits=[[0.0]])),
    ("logits: dtype", dict(logits=z(N, A).double())),
    ("logits: shape", dict(logits=z(N))),
    ("logits: strides", dict(logits=z(A, N).t())),
    ("actions: dtype", dict(actions=z(N, dtype=torch.int32))),
    ("actions: shape", dict(actions=z(N + 1, dtype=torch.int64))),
    ("offsets: expected a torch tensor", dict(offsets=[0, 3, 6])),
    ("offsets: shape", dict(offsets=z(2 * P, dtype=torch.int64))),
    ("offsets: shape", dict(offsets=z(0, dtype=torch.int64))),
    ("offsets: shape", dict(offsets=z(1, 3, dtype=torch.int64))),
    ("offsets: dtype", dict(offsets=z(2 * P + 1, dtype=torch.int32))),
    ("offsets: tensor is not contiguous", dict(offsets=z(4 * P + 2, dtype=torch.int64)[::2])),
    ("ref_logp: shape", dict(ref_logp=z(2 * P))),
    ("ref_logp: dtype", dict(ref_logp=z(N).half())),
    ("weights: shape", dict(weights=z(N))),
    ("weights: dtype", dict(weights=z(P, dtype=torch.bool))),
    ("mask: shape", dict(mask=torch.ones(N, A + 1, dtype=torch.bool))),
    ("beta", dict(beta=0.0)),
    ("beta", dict(beta=float("inf"))),
    ("beta", dict(beta=float("nan"))),
    ("beta", dict(beta="much")),
    ("smoothing", dict(smoothing=1.0)),
    ("smoothing", dict(smoothing=-0.1)),
    ("denominator", dict(denominator=-1.0)),
    ("denominator", dict(denominator=1e39)),
    ("denominator", dict(denominator=1e-60)),
])
def test_preferences_refuse(match, bad):
    _raises(match, policy.preference_gradient, **_args(**bad))
    _raises(match, policy.preference_loss, **_args(**bad))


def test_an_average_that_is_no_truth_value():
    class Odd:
        def __bool__(self):
            raise KeyError("neither")

    for bad in (Odd(), z(2)):
        _raises("average: ", policy.preference_gradient, **_args(average=bad))
        _raises("average: ", policy.preference_loss, **_args(average=bad))


def test_output_buffers_are_checked():
    ok = lambda **k: dict(_args(), out_stats=z(4), out_ratios=z(2 * P), dlogits=z(N, A), **k)
    _raises("out_stats: shape", pictura.pictura_preference_loss, **dict(ok(), out_stats=z(6)))
    _raises("out_ratios: shape", pictura.pictura_preference_loss, **dict(ok(), out_ratios=z(P)))
    _raises("dlogits: shape", pictura.pictura_preference_loss, **dict(ok(), dlogits=z(N, A + 1)))
    _raises("dlogits: dtype", pictura.pictura_preference_loss, **dict(ok(), dlogits=z(N, A).half()))


def test_host_tensors_are_refused_for_their_device():
    _raises("expected the HIP device", policy.preference_gradient, **_args())


def test_the_c_entry_refuses():
    L, ref = pictura._lib, ctypes.byref

    def call(ws=256, size=1 << 40, stats=64, ratios=64, dl=64, stride=A, logits=None, **over):
        l = pictura._Logits(64, 0, A, N, A, None, 0)
        for k, v in (logits or {}).items():
            setattr(l, k, v)
        p = pictura._Preferences(64, 64, 64, None, P, 0.1, 0.0, 0.0, 0)
        for k, v in over.items():
            setattr(p, k, v)
        return L.pictura_preference_loss(ref(l), ref(p), ws, size, stats, ratios, dl, stride, None)

    nan, inf = float("nan"), float("inf")
    for k in (dict(ws=None), dict(ws=128), dict(size=8), dict(stats=None), dict(stats=66), dict(ratios=None), dict(ratios=66), dict(dl=None),
              dict(dl=66), dict(stride=A - 1), dict(actions=None), dict(actions=68), dict(offsets=None), dict(offsets=68), dict(ref_logp=66),
              dict(weights=66), dict(pairs=-1), dict(pairs=(1 << 23) + 1), dict(beta=0.0), dict(beta=nan), dict(beta=inf), dict(smoothing=1.0),
              dict(smoothing=nan), dict(denominator=-1.0), dict(denominator=inf), dict(logits=dict(rows=-1)), dict(logits=dict(dtype=3)),
              dict(logits=dict(actions=0)), dict(logits=dict(stride=A - 1))):
        assert call(**k) == pictura.EINVAL, k
    out = ctypes.c_uint64()
    assert L.pictura_preference_loss_workspace(-1, 3, 1, ctypes.addressof(out)) == pictura.EINVAL
    assert L.pictura_preference_loss_workspace(1, 3, (1 << 23) + 1, ctypes.addressof(out)) == pictura.EINVAL
    assert L.pictura_preference_loss_workspace(1, 3, 1, None) == pictura.EINVAL


@pytest.mark.parametrize("name", ["ref_logp", "weights"])
def test_tensors_without_a_gradient_that_want_one(name):
    from paper_2607_26005_amd import policy
    from paper_2607_26005_amd.pictura import PicturaError
    a = dict(logits=torch.zeros(4, 3, requires_grad=True), actions=torch.zeros(4, dtype=torch.int64),
             offsets=torch.tensor([0, 2, 4]), ref_logp=torch.zeros(4), weights=torch.ones(1))
    a[name].requires_grad_()
    with pytest.raises(PicturaError, match=f"{name}: .*no gradient"):
        policy.preference_loss(**a)
    with torch.no_grad(), pytest.raises(PicturaError, match="expected the HIP device"):   # (the next check)
        policy.preference_loss(**a)
