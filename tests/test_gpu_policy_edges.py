"""Draws, losses and steps at the ends of what their arguments allow."""
import numpy as np
import pytest

from tests import policy_oracle as PO

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def mods():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no HIP device")
    from paper_2607_26005_amd import policy
    return torch, policy


def _draw_by_rule(torch, x, w, u, top_k=0, top_p=1.0, min_p=0.0):
    """The drawing rule in whole numbers, given the weights (int64) of the logits."""
    one = 1 << 31
    cut = lambda v: (v.clamp(0.0, 1.0 - 2.0 ** -24) * float(one)).to(torch.int64)
    share = lambda W, m: (W >> 32) * m * 2 + ((W & 0xFFFFFFFF) * m >> 31)
    order = x.sort(dim=1, descending=True, stable=True).indices
    ws = w.gather(1, order)
    if top_k > 0:
        ws[:, top_k:] = 0
    if top_p < 1:
        need = share(ws.sum(1, keepdim=True), cut(torch.tensor(top_p, dtype=torch.float32, device=x.device))).clamp_min(1)
        ws = ws * (ws.cumsum(1) - ws < need)
    ws = ws * (ws >= int(np.ceil(np.float32(min_p) * np.float32(one))))
    c = torch.zeros_like(w).scatter_(1, order, ws).cumsum(1)
    act = (c <= share(c[:, -1:], cut(u)[:, None])).sum(1)
    return act, torch.zeros_like(w).scatter_(1, order, ws).gather(1, act[:, None])[:, 0], c[:, -1]


@pytest.mark.parametrize("N, A", [(9, 1), (9, 12), (9, 40), (9, 300), (300, 300), (300, 2000), (9, 5000), (300, 5000), (4, 40000),
                                  (4, 80000)])
def test_an_infinite_temperature_draws_evenly(mods, N, A):
    # every allowed action of finite logit weighs 2^31, whatever the logits: the rest of
    # the rule (order, filters, the draw) is unchanged
    torch, policy = mods
    g = torch.Generator().manual_seed(A)
    for dtype in (torch.float32, torch.bfloat16):
        x = (torch.randn(N, A, generator=g) * 3).to(dtype).cuda()
        mask = (torch.rand(N, A, generator=g) < 0.7).cuda()
        mask[:, 0] = True
        if A > 1:
            x[:, 1] = float("-inf")
        u = torch.rand(N, generator=g).cuda()
        for m in (None, mask):
            z = x.float() if m is None else x.float().masked_fill(~m, -float("inf"))
            w = (z > -float("inf")).long() << 31
            for how in (dict(), dict(top_k=3), dict(top_k=A // 2), dict(top_p=0.4), dict(top_k=700, top_p=0.6), dict(min_p=1.0, top_p=0.9)):
                want, mine, total = _draw_by_rule(torch, z, w, u, **how)
                per_row = torch.full((N,), float("inf"), device="cuda")
                for t in (float("inf"), per_row):
                    act, logp = policy.sample_actions(x, u, mask=m, temperature=t, **how)
                    assert torch.equal(act, want), (dtype, how, (act != want).nonzero().flatten().tolist())
                    # (the logarithm of the same quotient: a unit of it)
                    ref = (mine.double() / total.double()).log()
                    assert ((logp.double() - ref).abs() <= 2.0 ** -22 * ref.abs() + 2.0 ** -23).all(), how
                # one such row leaves the others as they are
                per_row[1:] = 0.8
                act, logp = policy.sample_actions(x, u, mask=m, temperature=per_row, **how)
                plain, plogp = policy.sample_actions(x, u, mask=m, temperature=0.8, **how)
                assert act[0] == want[0] and torch.equal(act[1:], plain[1:]) and torch.equal(logp[1:], plogp[1:])


def _decisions(torch, N, A, dtype, seed):
    """Logits and a batch of decisions, log-ratios away from the clip's edges."""
    g = torch.Generator().manual_seed(seed)
    rnd = lambda *s: torch.randn(*s, generator=g)
    z = (rnd(N, A) * 1.5).to(dtype)
    b = dict(actions=torch.randint(0, A, (N,), generator=g), advantages=rnd(N) + 0.2, values=rnd(N))
    b["returns"] = b["values"] + rnd(N)
    diff = rnd(N).double() * 0.3
    r = diff.exp()
    diff = torch.where(((r - 0.8).abs() < 1e-3) | ((r - 1.2).abs() < 1e-3), torch.full_like(diff, 0.01), diff)
    b["old_logp"] = (z.double().log_softmax(1).gather(1, b["actions"][:, None])[:, 0] - diff).float()
    return z, b


def _oracle(z, b, **kw):
    return PO.policy_loss(z.float().numpy(), *(b[k].numpy() for k in ("values", "actions", "old_logp", "advantages", "returns")), **kw)


# what fp32 arithmetic before a rounding costs (as in tests/test_gpu_policy.py), and the
# rounding: half a unit, in fp16 at least half of 2^-24
ROUND = {"float32": (2.0 ** -16, 0.0), "bfloat16": (2.0 ** -16 + 2.0 ** -8, 0.0), "float16": (2.0 ** -16 + 2.0 ** -11, 2.0 ** -25)}


@pytest.mark.parametrize("dtype", ["float16", "bfloat16", "float32"])
@pytest.mark.parametrize("N, A", [(300, 12), (4096, 12), (1500, 40), (700, 999), (33, 16381), (5, 80000)])
def test_a_loss_scale_lifts_what_the_logits_type_could_not_hold(mods, N, A, dtype):
    # the gradient under a scale is the 64-bit one times the scale, rounded once
    torch, policy = mods
    z, b = _decisions(torch, N, A, getattr(torch, dtype), N + A)
    _, dz, dv = _oracle(z, b)
    c = {k: v.cuda() for k, v in b.items()}
    for scale in (2.0 ** 16, 2.0 ** 13, 1.0):
        x, v = z.cuda().requires_grad_(), c["values"].clone().requires_grad_()
        loss, stats = policy.policy_loss(x, v, c["actions"], c["old_logp"], c["advantages"], c["returns"])
        (scale * loss).backward()
        assert x.grad.dtype == x.dtype and stats.dtype == loss.dtype == torch.float32
        want, got = dz * scale, x.grad.double().cpu().numpy()
        rel, least = ROUND[dtype]
        assert (np.abs(got - want) <= rel * np.abs(want) + 2.0 ** -20 * np.abs(want).max() + least).all()
        assert (np.abs(v.grad.double().cpu().numpy() - dv * scale) <= 2.0 ** -20 * np.abs(dv * scale).max()).all()


@pytest.mark.parametrize("A", [1, 5, 12, 40, 300, 5000, 80000])
@pytest.mark.parametrize("exponent", [-140, -127, -126, -90, -60])
def test_loss_at_the_smallest_temperatures(mods, A, exponent):
    # the softmax is one at the largest logit and zero elsewhere; in fp32 as in 64 bits
    # no gradient is left of it, the ratio of any other action is 0, values learn as ever.
    # (Row 0 may have drawn another action, of log-probability (z - top) / T: a number beyond
    # where the oracle's exponential, and so its logarithm, has one.)
    torch, policy = mods
    N, T = 9, 2.0 ** exponent
    z, b = _decisions(torch, N, A, torch.float32, A)
    b["actions"][1:] = z[1:].argmax(1)
    b["old_logp"] = torch.randn(N, generator=torch.Generator().manual_seed(1)) * 0.3
    stats, dz, dv = _oracle(z, b, temperature=T, entropy_coef=0.3)
    assert (dz == 0).all() and np.isfinite(stats[[0, 1, 2, 3, 5]]).all()
    c = {k: v.cuda() for k, v in b.items()}
    out = policy.policy_gradient(z.cuda(), c["values"], c["actions"], c["old_logp"], c["advantages"], c["returns"], temperature=T,
                                 entropy_coef=0.3)
    got = out.stats.cpu().double().numpy()
    rest = [0, 1, 2, 3, 5]
    assert np.abs(got[rest] - stats[rest]).max() <= 2.0 ** -16 * max(1.0, np.abs(stats[rest]).max()), (got, stats)
    top = z.gather(1, b["actions"][:, None])[:, 0].double() - z.max(1).values.double()
    diff = (top / T - b["old_logp"].double()).numpy()
    with np.errstate(over="ignore"):
        kl = np.where(np.abs(diff.astype(np.float32)) < np.inf, np.expm1(diff) - diff, np.inf).mean()
    assert got[4] == kl if kl == np.inf else abs(got[4] - kl) <= 2.0 ** -16 * max(1.0, kl), (got[4], kl)
    assert (out.dlogits == 0).all(), out.dlogits[out.dlogits != 0]
    assert (np.abs(out.dvalues.cpu().double().numpy() - dv) <= 2.0 ** -20 * np.abs(dv).max()).all()


@pytest.mark.parametrize("A", [12, 40, 300, 80000])
def test_a_part_whose_weights_cancel_still_counts(mods, A):
    # weights of both signs that add up to 0 in one part of a minibatch: by the denominator
    # of the whole its rows count like any others; without one there is no mean to take
    torch, policy = mods
    N = 6
    z, b = _decisions(torch, N, A, torch.float32, 2 * A)
    w = torch.tensor([0.5, -0.5, 1.25, -1.0, -0.25, 0.0])
    c = {k: v.cuda() for k, v in b.items()}
    run = lambda **kw: policy.policy_gradient(z.cuda(), c["values"], c["actions"], c["old_logp"], c["advantages"], c["returns"],
                                              weights=w.cuda(), **kw)
    stats, dz, dv = _oracle(z, b, weights=w.numpy(), denominator=8.0)
    out = run(denominator=8.0)
    assert np.abs(dz).max() > 1e-3
    assert np.abs(out.stats.cpu().double().numpy() - stats).max() <= 2.0 ** -16
    got = out.dlogits.cpu().double().numpy()
    assert (np.abs(got - dz) <= 2.0 ** -16 * np.abs(dz) + 2.0 ** -20 * np.abs(dz).max()).all()
    assert (np.abs(out.dvalues.cpu().double().numpy() - dv) <= 2.0 ** -20 * np.abs(dv).max()).all()
    out = run()
    assert (out.stats == 0).all() and (out.dlogits == 0).all() and (out.dvalues == 0).all()


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("eps", [0.0, 2.0 ** -140, 1e-30, 1e-20, 1e-15])
def test_steps_with_next_to_no_epsilon(mods, bits, eps):
    # v of gradients down to 1e-19 is 1e-40, a number of 17 bits in fp32: its root is off by
    # 2^-18 of itself, and with it the update
    torch, policy = mods
    how = dict(lr=1e-3, betas=(0.9, 0.99), weight_decay=0.0)
    g = torch.Generator().manual_seed(0)
    n = 5000
    sizes = 10.0 ** (torch.rand(n, generator=g) * 18 - 19)
    grad = sizes * torch.where(torch.rand(n, generator=g) < 0.5, -1.0, 1.0)
    if eps > 0:
        grad[256:700] = 0.0                                  # whole blocks of nothing: 0 / eps
    p = torch.nn.Parameter(torch.zeros(n).cuda())
    policy.AdamW([p], **how, eps=eps, bits=bits).step(grads=[grad.cuda()])
    eps32 = float(np.float32(eps))
    want = PO.adamw(np.zeros(n), grad.double().numpy(), np.zeros(n), np.zeros(n), 1, how["lr"], how["betas"], eps32, 0.0)[0]
    got = p.detach().double().cpu().numpy()
    assert (np.abs(got - want) <= 2.0 ** -16 * how["lr"]).all(), np.abs(got - want).max() / how["lr"]


@pytest.mark.parametrize("A", [12, 40, 300, 5000, 80000])
@pytest.mark.parametrize("exponent", [-145, -127, -100, -65, -64, -63, 63, 64, 65, 100, 122])
def test_temperatures_of_any_size_draw_by_their_quotients(mods, A, exponent):
    # logits as large as the temperature: the correctly rounded quotient, to the bit
    torch, policy = mods
    N, g = 8, torch.Generator().manual_seed(A)
    for T in (2.0 ** exponent, float(np.float32(1.37 * 2.0 ** exponent))):
        x = (torch.randn(N, A, generator=g).double() * 2.5 * T).float().cuda()
        u = torch.rand(N, generator=g).cuda()
        t = torch.full((N, 1), T, dtype=torch.float32, device="cuda")
        w = (((x - x.amax(1, keepdim=True)) / t).exp() * 2.0 ** 31).round().to(torch.int64)
        for how in (dict(), dict(top_k=7), dict(top_p=0.8), dict(top_k=400, top_p=0.5), dict(min_p=0.3)):
            want, mine, total = _draw_by_rule(torch, x, w, u, **how)
            act, logp = policy.sample_actions(x, u, temperature=T, **how)
            assert torch.equal(act, want), (T, how, (act != want).nonzero().flatten().tolist())
            ref = (mine.double() / total.double()).log()
            assert ((logp.double() - ref).abs() <= 2.0 ** -22 * ref.abs() + 2.0 ** -23).all(), how
