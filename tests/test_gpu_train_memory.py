"""The policy that remembers, as it is used: acting step by step, learning from whole
rollouts and from pairs of agents (paper_2607_26005_amd/train_policy.py, memory.MemoryLayer)."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def device():
    if not torch.cuda.is_available():
        pytest.skip("no HIP device")


@pytest.fixture
def trainer():
    from paper_2607_26005_amd import train_policy as tp
    made = []

    def make(**k):
        made.append(tp.Trainer(worlds=1, seed=1, **k))
        return made[-1]

    yield make
    for t in made:
        t.close()


def _layers(width, count, seed=0):
    from paper_2607_26005_amd import memory
    torch.manual_seed(seed)
    return [memory.MemoryLayer(width).cuda() for _ in range(count)]


def _whole(layers, x, states, resets):
    residual, after = None, []
    for layer, s in zip(layers, states):
        x, residual, last = layer(x, residual, s, resets)
        after.append(last)
    return x + residual, after


def test_steps_are_the_sequence():
    layers = _layers(48, 3)
    gen = torch.Generator().manual_seed(1)
    x = torch.randn(5, 19, 48, generator=gen).cuda()
    resets = (torch.rand(5, 19, generator=gen) < 0.2).cuda()
    states = [torch.randn(5, 48, generator=gen).cuda() for _ in layers]
    with torch.no_grad():
        want, after = _whole(layers, x, states, resets)
    held = [s.clone() for s in states]
    for t in range(19):
        y, residual = x[:, t], None
        for layer, s in zip(layers, held):
            y, residual = layer.step(y, residual, s, resets[:, t])
        # (matrix products of other shapes add up in another order: 48 terms, twice a layer)
        assert torch.allclose(y + residual, want[:, t], rtol=1e-4, atol=1e-4), t
    assert all(torch.allclose(a, b, rtol=1e-4, atol=1e-4) for a, b in zip(held, after))


def test_gradients_of_layers_against_differences():
    layers = _layers(16, 2)
    gen = torch.Generator().manual_seed(2)
    x = torch.randn(3, 600, 16, generator=gen).cuda()
    resets = (torch.rand(3, 600, generator=gen) < 0.01).cuda()
    states = [torch.randn(3, 16, generator=gen).cuda() for _ in layers]
    w = torch.randn(3, 600, 16, generator=gen).cuda().double() / 40
    params = [p for layer in layers for p in layer.parameters()]
    f = lambda: (_whole(layers, x, states, resets)[0].double() * w).sum()
    grads = torch.autograd.grad(f(), params)
    assert all(g.isfinite().all() for g in grads)
    for p, g in zip(params, grads):
        d = torch.randn(p.shape, generator=gen).cuda()
        d /= d.norm()
        ends = []
        with torch.no_grad():
            for sign in (1, -1):
                p.add_(d, alpha=sign * 0.01)
                ends.append(f())
                p.sub_(d, alpha=sign * 0.01)
        got, want = (g.double() * d).sum(), (ends[0] - ends[1]) / 0.02
        # fp32 values off by 1e-6 of about 30,000 terms of 1/40 (in quadrature 4e-6) over the step, and
        # step^2 / 6 of the third derivative
        assert abs(got - want) <= 1e-3 + 1e-2 * g.double().norm(), (tuple(p.shape), got.item(), want.item())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_layers_under_autocast(dtype):
    """Products in 16 bits, the stream between the layers in its own type: bit for bit what the same
    layers do by hand."""
    from paper_2607_26005_amd import memory
    layers = _layers(48, 3)
    gen = torch.Generator().manual_seed(4)
    x = torch.randn(2, 9, 48, generator=gen).cuda().requires_grad_()
    dy = torch.randn(2, 9, 48, generator=gen).cuda()
    params = [x] + [p for layer in layers for p in layer.parameters()]

    def by_hand(x):
        cut = lambda m, t: torch.nn.functional.linear(t.to(dtype), m.weight.to(dtype), m.bias.to(dtype))
        stream, y = None, x
        for layer in layers:
            if stream is None:
                normed, stream = memory.rms_norm(y, layer.norm), y
            else:
                normed, stream = memory.rms_norm(y.float(), layer.norm, stream)
            gates, inputs = cut(layer.project, normed).chunk(2, -1)
            y = cut(layer.out, memory.gated_scan(gates, inputs, torch.zeros(2, 48, device="cuda"))[0])
        return y, stream

    y, stream = by_hand(x)
    want = torch.autograd.grad((y.float() + stream, ), params, dy)
    with torch.autocast("cuda", dtype=dtype):
        got, went = x, None
        for layer in layers:
            got, went, _ = layer(got, went, torch.zeros(2, 48, device="cuda"))
    assert got.dtype == dtype and went.dtype == torch.float32 and torch.equal(got, y) and torch.equal(went, stream)
    grads = torch.autograd.grad((got.float() + went, ), params, dy)
    assert all(map(torch.equal, grads, want))
    # and step by step (matrix products of other shapes add up in another order: a unit of the type
    # in each of six products of values of some 2)
    states = [torch.zeros(2, 48, device="cuda") for _ in layers]
    codes = [layer.quantized() for layer in layers]
    for t in range(9):
        for how in (None, codes):
            held = states if how is None else [s.clone() for s in states]
            with torch.autocast("cuda", dtype=dtype):
                z, r = x.detach()[:, t], None
                for i, layer in enumerate(layers):
                    z, r = layer.step(z, r, held[i], None, how and how[i])
            assert z.dtype == dtype and r.dtype == torch.float32
            if how is None:
                assert torch.allclose(z.float() + r, (y.float() + stream)[:, t], atol=24 * torch.finfo(dtype).eps)
            else:
                assert z.isfinite().all() and r.isfinite().all()


def test_projection_in_8_bits():
    from paper_2607_26005_amd import memory
    layer, = _layers(64, 1)
    gen = torch.Generator().manual_seed(3)
    x, r = torch.randn(32, 64, generator=gen).cuda(), torch.randn(32, 64, generator=gen).cuda()
    y, s = memory.rms_norm(x, layer.norm, r)
    codes = layer.quantized()
    held = memory.rms_norm_8bit(x, layer.norm, r)
    assert torch.equal(held.sum, s)
    w = layer.project.weight.detach().double()
    # e4m3 is off by half a step, 2^-4 of a value, or 2^-10 of the scale among the smallest; a weight's
    # scale is off by a unit of fp32 more
    ey = torch.maximum(y.double().abs() * 2.0 ** -4, held.scales.double()[:, None] * 2.0 ** -10)
    ew = torch.maximum(w.abs() * 2.0 ** -4, codes[1].double().t() * 2.0 ** -10) * (1 + 2.0 ** -20)
    exact = y.double() @ w.t()
    bound = ey @ w.abs().t() + y.double().abs() @ ew.t() + ey @ ew.t()
    got = torch._scaled_mm(held.codes, codes[0].t(), scale_a=held.scales[:, None], scale_b=codes[1], out_dtype=torch.bfloat16)
    limit = bound + (exact.abs() + bound) * 2.0 ** -8 + 1e-4
    assert ((got.double() - exact).abs() <= limit).all()
    a, b = torch.zeros(32, 64, device="cuda"), torch.zeros(32, 64, device="cuda")
    out, stream = layer.step(x, r, a, None, codes)
    want, _ = layer.step(x, r, b)
    assert torch.equal(stream, s) and (a - b).abs().max() < 0.3 and torch.isfinite(out).all() and out.shape == want.shape


@pytest.mark.parametrize("episode", [0, 3])
def test_acting_and_learning(trainer, episode):
    from paper_2607_26005_amd import policy, train_policy as tp
    t = trainer(layers=2, episode=episode)
    before = [p.detach().clone() for p in t.net.parameters()]
    for k in range(2):
        batch = t.remembered_rollout(5)
        seen, resets, states, actions, logp, values, adv, returns = batch
        n = t.agents.x.numel()
        assert len(seen) == 5 and actions.shape == logp.shape == values.shape == adv.shape == returns.shape == (n, 5)
        assert resets.shape == (n, 5) and resets[0].tolist() == [(5 * k + i) % (episode or 99) == 0 for i in range(5)]
        assert ((actions >= 0) & (actions < tp.ACTIONS)).all()
        # the sequence gives the log-probabilities that the steps acted with
        with torch.no_grad():
            out = t.net.sequence(seen, states, resets)
        want = out[..., :tp.ACTIONS].log_softmax(2).gather(2, actions[..., None])[..., 0]
        assert torch.allclose(logp, want, atol=1e-3) and torch.allclose(values, out[..., tp.ACTIONS], atol=1e-3)
        stats, liked = t.remembered_update(batch, epochs=1, prefer=0.1)
        assert torch.isfinite(stats).all() and torch.isfinite(liked).all()
        # the policy is still the one that acted: nothing is preferred yet
        assert abs(liked[0].item() - math.log(2)) < 1e-3 and abs(dict(zip(policy.POLICY_STATS, stats.tolist()))["approx_kl"]) < 1e-4
    assert all(torch.isfinite(p).all() for p in t.net.parameters())
    moved = [bool((p != b).any()) for p, b in zip(t.net.parameters(), before)]
    assert all(moved), [n for (n, _), m in zip(t.net.named_parameters(), moved) if not m]


def test_acting_in_8_bits(trainer):
    t = trainer(layers=2, act_bits=8, bits=8)
    batch = t.remembered_rollout(4)
    stats, liked = t.remembered_update(batch, epochs=2, prefer=0.5)
    assert torch.isfinite(stats).all() and torch.isfinite(liked).all()
    assert all(torch.isfinite(p).all() for p in t.net.parameters())


def test_a_policy_without_a_memory_has_none(trainer):
    t = trainer()
    assert not t.states and not any(n.startswith("memory") or n == "norm" for n, _ in t.net.named_parameters())
