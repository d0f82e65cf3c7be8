"""The AdamW step over many tensors, with moments in 32 and in 8 bits, against a
64-bit implementation (tests/policy_oracle.py)."""
import numpy as np
import pytest

from tests import policy_oracle as PO

pytestmark = pytest.mark.gpu

HOW = dict(lr=3e-3, betas=(0.9, 0.99), eps=1e-8, weight_decay=0.1)
SIZES = (1, 3, 255, 256, 257, 511, 1024, 4095, 4096, 4097, 12289, 70001)


@pytest.fixture(scope="module")
def mods():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no HIP device")
    from paper_2607_26005_amd import policy
    return torch, policy


def _params(torch, sizes, dtype, seed, offset=0):
    """Parameters cut from one storage, `offset` elements apart: any alignment."""
    g = torch.Generator().manual_seed(seed)
    whole = (torch.randn(sum(sizes) + offset * (len(sizes) + 1), generator=g) * 0.1).to(dtype).cuda()
    out, at = [], offset
    for n in sizes:
        out.append(torch.nn.Parameter(whole[at:at + n]))
        at += n + offset
    return out


def _grads(torch, sizes, dtype, seed, offset=0):
    return [p.data * 10 ** (i % 4 - 3) for i, p in enumerate(_params(torch, sizes, dtype, seed, offset))]


def _f64(t):
    return t.detach().double().cpu().numpy().reshape(-1)


# fp32: the products, sums, root and quotient of one element, half a unit each
EPS32 = 2.0 ** -20
UNIT = {"float32": 2.0 ** -24, "bfloat16": 2.0 ** -8, "float16": 2.0 ** -11}


@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("gtype", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("offset", [0, 1, 3])
def test_steps_match_float64(mods, dtype, gtype, offset):
    torch, policy = mods
    ps = _params(torch, SIZES, getattr(torch, dtype), 1, offset)
    opt = policy.AdamW(ps, **HOW)
    for step in range(1, 4):
        # each step from the device's own state, so errors do not add up
        gs = _grads(torch, SIZES, getattr(torch, gtype), 10 + step, offset)
        before = [(_f64(p), *[_f64(t) for t in ((opt.state[p]["exp_avg"], opt.state[p]["exp_avg_sq"]) if opt.state.get(p)
                                               else (torch.zeros(p.numel()),) * 2)]) for p in ps]
        opt.step(grads=gs)
        for p, g, (p0, m0, v0) in zip(ps, gs, before):
            rp, rm, rv = PO.adamw(p0, _f64(g), m0, v0, step, HOW["lr"], HOW["betas"], HOW["eps"], HOW["weight_decay"])
            m, v = _f64(opt.state[p]["exp_avg"]), _f64(opt.state[p]["exp_avg_sq"])
            # (m's two terms may cancel)
            assert (np.abs(m - rm) <= EPS32 * (np.abs(m0) + np.abs(_f64(g)))).all()
            assert (np.abs(v - rv) <= EPS32 * rv).all()
            move = np.abs(rp - p0) + HOW["lr"]
            assert (np.abs(_f64(p) - rp) <= (UNIT[dtype] + 2.0 ** -23) * np.abs(rp) + 2.0 ** -18 * move
                    + (2.0 ** -25 if dtype == "float16" else 0)).all()


def test_matches_torch_adamw_over_steps(mods):
    torch, policy = mods
    ps = _params(torch, (5, 300, 4097), torch.float32, 2)
    qs = [torch.nn.Parameter(p.detach().clone()) for p in ps]
    a = policy.AdamW(ps, **HOW)
    b = torch.optim.AdamW(qs, **HOW, foreach=False)
    for step in range(20):
        for p, q, g in zip(ps, qs, _grads(torch, (5, 300, 4097), torch.float32, 50 + step)):
            p.grad, q.grad = g.clone(), g.clone()
        a.step()
        b.step()
    for p, q in zip(ps, qs):
        assert torch.allclose(p, q, rtol=1e-5, atol=1e-6)


@pytest.mark.parametrize("bits", [32, 8])
def test_clipping_to_a_common_norm(mods, bits):
    torch, policy = mods
    for scale, max_norm in ((100.0, 0.5), (1e-4, 0.5), (0.0, 0.5), (1.0, 0.0)):
        ps = _params(torch, SIZES, torch.float32, 3)
        gs = [(g * scale).to((torch.float32, torch.bfloat16, torch.float16)[i % 3]) for i, g in
              enumerate(_grads(torch, SIZES, torch.float32, 4))]
        opt = policy.AdamW(ps, **HOW, bits=bits, max_norm=max_norm)
        before = [_f64(p) for p in ps]
        opt.step(grads=gs)
        norm = np.sqrt(sum((_f64(g) ** 2).sum() for g in gs))
        assert abs(opt.grad_norm.item() - norm) <= 2.0 ** -23 * norm
        factor = min(1.0, max_norm / (norm + 1e-6))
        for p, g, p0 in zip(ps, gs, before):
            rp = PO.adamw(p0, _f64(g), 0 * p0, 0 * p0, 1, HOW["lr"], HOW["betas"], HOW["eps"], HOW["weight_decay"], factor)[0]
            assert (np.abs(_f64(p) - rp) <= 2.0 ** -22 * np.abs(rp) + 2.0 ** -16 * HOW["lr"]).all()


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("offset", [0, 1, 3])
def test_eight_bit_steps_match_float64(mods, dtype, offset):
    torch, policy = mods
    ps = _params(torch, SIZES, getattr(torch, dtype), 5, offset)
    opt = policy.AdamW(ps, **HOW, bits=8)
    for step in range(1, 4):
        gs = _grads(torch, SIZES, torch.float32, 20 + step, offset)
        before = []
        for p in ps:
            s = opt.state.get(p)
            z = np.zeros(p.numel())
            before.append((_f64(p), *((PO.moment_values(_f64(s["exp_avg"]), _f64(s["exp_avg_scale"]), False),
                                       PO.moment_values(_f64(s["exp_avg_sq"]), _f64(s["exp_avg_sq_scale"]), True)) if s else (z, z))))
        opt.step(grads=gs)
        got_m, got_v = opt.moments()
        for p, g, (p0, m0, v0), gm, gv in zip(ps, gs, before, got_m, got_v):
            rp, rm, rv = PO.adamw(p0, _f64(g), m0, v0, step, HOW["lr"], HOW["betas"], HOW["eps"], HOW["weight_decay"])
            s = opt.state[p]
            move = np.abs(rp - p0) + HOW["lr"]
            assert (np.abs(_f64(p) - rp) <= (UNIT[dtype] + 2.0 ** -22) * np.abs(rp) + 2.0 ** -16 * move).all()
            for code, scale, ref, val, second in ((s["exp_avg"], s["exp_avg_scale"], rm, gm, False),
                                                  (s["exp_avg_sq"], s["exp_avg_sq_scale"], rv, gv, True)):
                q, sc = PO.moment_positions(ref, second)
                # the code is the nearest to where the value lies: half a step, and fp32's
                # error (m's terms may cancel, so it is that of the block's largest: less
                # than 2^-16 of it, whose root on 127 steps is half of one near zero)
                c = _f64(code)
                off = np.abs(c - np.where(second & (ref > 0), np.maximum(q, 1), q))
                assert (off <= 0.51 if second else off <= 1.0).all() and (off <= 0.51).mean() > 0.99, off.max()
                terms = rv if second else np.abs(m0) + np.abs(_f64(g))   # (as m itself: its terms may cancel)
                assert (np.abs(_f64(scale) - sc) <= EPS32 * PO.moment_positions(terms, second)[1]).all()
                want = PO.moment_values(c, _f64(scale), second)
                assert (np.abs(_f64(val) - want) <= 2.0 ** -21 * np.abs(want)).all()


def test_eight_bit_moments_follow_the_fp32_ones(mods):
    # gradients of spread scales over 200 steps: the update keeps within a tenth of the fp32 one's norm
    torch, policy = mods
    n = 256 * 40 + 17
    g = torch.Generator().manual_seed(0)
    scale = (torch.randn(n, generator=g) * 0.5).exp() * 1e-3
    a, b = (torch.nn.Parameter(torch.zeros(n).cuda()) for _ in range(2))
    kw = dict(lr=1e-3, betas=(0.9, 0.999), weight_decay=0.0)
    full, small = policy.AdamW([a], **kw), policy.AdamW([b], **kw, bits=8)
    for _ in range(200):
        grad = ((torch.randn(n, generator=g) + 0.3) * scale).cuda()
        full.step(grads=[grad])
        small.step(grads=[grad])
    assert (a - b).norm() < 0.1 * a.norm()


@pytest.mark.parametrize("bits", [32, 8])
def test_zero_and_nonfinite_gradients(mods, bits):
    torch, policy = mods
    n = 600
    p = torch.nn.Parameter(torch.ones(n).cuda())
    opt = policy.AdamW([p], **HOW, bits=bits)
    opt.step(grads=[torch.zeros(n).cuda()])
    keep = np.float32(1 - HOW["lr"] * HOW["weight_decay"])
    assert (p == float(keep)).all()                       # decay alone; 0 / (0 + eps) is 0
    opt.step(grads=[torch.full((n,), 1e-30).cuda()])      # squares that vanish
    assert p.isfinite().all()
    g = torch.zeros(n)
    g[300] = float("nan")
    g[590] = float("inf")
    opt.step(grads=[g.cuda()])
    bad = ~p.isfinite().cpu()
    assert bad[300] and bad[590] and bad.sum() == 2       # the parameter goes loudly where the gradient did
    if bits == 8:
        m, v = opt.moments()
        assert m[0][256:512].isnan().all() and v[0][256:512].isnan().all() and m[0][:256].isfinite().all()
    opt2 = policy.AdamW([p], **HOW, max_norm=1.0)
    opt2.step(grads=[g.cuda()])
    assert opt2.grad_norm.isnan() and p.isnan().all()     # a norm of NaN is not hidden


def test_many_tensors_and_groups(mods):
    # more tensors than one launch takes, empty ones among them, two groups, some without a gradient
    torch, policy = mods
    sizes = [(i * 37) % 700 for i in range(150)]
    ps, qs = _params(torch, sizes, torch.float32, 7), _params(torch, sizes, torch.float32, 7)
    groups = lambda x: [dict(params=x[:80], lr=1e-2), dict(params=x[80:], weight_decay=0.0)]
    a, b = policy.AdamW(groups(ps), **HOW), torch.optim.AdamW(groups(qs), **HOW, foreach=False)
    for step in range(3):
        for i, (p, q, g) in enumerate(zip(ps, qs, _grads(torch, sizes, torch.float32, 70 + step))):
            p.grad = q.grad = None if i % 11 == step else g
        a.step()
        b.step()
    for p, q in zip(ps, qs):
        assert torch.allclose(p, q, rtol=1e-5, atol=1e-6)


@pytest.mark.parametrize("bits", [32, 8])
def test_checkpoint_of_the_optimizer(mods, bits):
    torch, policy = mods
    import copy
    sizes = (300, 7)
    ps = _params(torch, sizes, torch.bfloat16, 8)
    opt = policy.AdamW(ps, **HOW, bits=bits)
    opt.step(grads=_grads(torch, sizes, torch.float32, 1))
    held = copy.deepcopy(opt.state_dict())
    qs = [torch.nn.Parameter(p.detach().clone()) for p in ps]
    other = policy.AdamW(qs, **HOW, bits=bits)
    other.load_state_dict(held)
    for o in (opt, other):
        o.step(grads=_grads(torch, sizes, torch.float32, 2))
    for p, q in zip(ps, qs):
        assert torch.equal(p, q)
        assert all(torch.equal(opt.state[p][k], other.state[q][k]) for k in opt.state[p] if k != "step")
        assert opt.state[p]["step"] == other.state[q]["step"] == 2


def test_step_in_a_graph(mods):
    # the norm, its factor and the update replay with new gradients (step number and rate are the captured ones)
    torch, policy = mods
    from paper_2607_26005_amd import pictura
    sizes = (5000, 33)
    ps, qs = _params(torch, sizes, torch.float32, 9), _params(torch, sizes, torch.float32, 9)
    gs = _grads(torch, sizes, torch.float32, 9)
    opts = [policy.AdamW(x, **HOW, max_norm=0.1) for x in (ps, qs)]
    for o in opts:
        o.step(grads=gs)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        opts[0].step(grads=gs)
    for k in range(3):
        for g in gs:
            g.copy_(torch.randn(g.shape, generator=torch.Generator().manual_seed(k)))
        graph.replay()
        torch.cuda.synchronize()
        for q in qs:
            opts[1].state[q]["step"] = 1
        opts[1].step(grads=gs)
        torch.cuda.synchronize()
        for p, q in zip(ps, qs):
            assert torch.equal(p, q), k


def test_hooks_and_schedulers(mods):
    # hooks around a step run, and a scheduler's rate is the one that is used
    torch, policy = mods
    p = torch.nn.Parameter(torch.ones(10).cuda())
    opt = policy.AdamW([p], lr=1e-2, weight_decay=0.0)
    sched = torch.optim.lr_scheduler.CosineAnnealingLR(opt, T_max=4)
    seen = []
    pre = opt.register_step_pre_hook(lambda o, a, k: seen.append("pre"))
    opt.register_step_post_hook(lambda o, a, k: seen.append("post"))
    rates = []
    for _ in range(3):
        p.grad = torch.ones(10).cuda()
        before = p.detach().clone()
        opt.step()
        rates.append((before - p).mean().item())   # a constant gradient moves by the rate
        sched.step()
    assert seen == ["pre", "post"] * 3
    want = [1e-2 * (1 + np.cos(np.pi * k / 4)) / 2 for k in range(3)]
    assert np.allclose(rates, want, rtol=1e-4)
    pre.remove()
    opt.zero_grad()
    assert p.grad is None
