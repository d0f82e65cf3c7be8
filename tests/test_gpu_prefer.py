"""The preference loss on the device against its 64-bit form on the host
(tests/preference_oracle.py)."""
import math

import pytest
import torch

from tests import preference_oracle as O

pytestmark = pytest.mark.gpu

DTYPES = [torch.float32, torch.bfloat16, torch.float16]


@pytest.fixture(autouse=True)
def device():
    if not torch.cuda.is_available():
        pytest.skip("no HIP device")


def _inputs(lengths, A, dtype=torch.float32, seed=0, pad=0, mask=0.0, unused=0.0, scale=2.0, outside=0):
    """logits, actions, offsets, ref_logp, mask; the sequences have these lengths."""
    g = torch.Generator().manual_seed(seed)
    N = sum(lengths) + 2 * outside
    logits = torch.zeros(N, A + pad, dtype=dtype, device="cuda")[:, :A].copy_(torch.randn(N, A, generator=g) * scale)
    m = None
    if mask:
        m = torch.rand(N, A, generator=g) < mask
        m[torch.arange(N), torch.randint(A, (N,), generator=g)] = True
    z = logits.cpu().double() if m is None else logits.cpu().double().masked_fill(~m, -math.inf)
    actions = (z - (-torch.rand(N, A, generator=g).double().clamp_min(1e-20).log()).log()).argmax(1)
    ref = z.log_softmax(1).gather(1, actions[:, None])[:, 0] + torch.randn(N, generator=g) * 0.2
    actions = torch.where(torch.rand(N, generator=g) < unused, torch.full_like(actions, -1), actions)
    offsets = torch.tensor([0] + lengths).cumsum(0) + outside
    return logits, actions.cuda(), offsets.cuda(), ref.float().cuda(), None if m is None else m.cuda()


def _check(logits, actions, offsets, ref=None, **k):
    from paper_2607_26005_amd import policy
    got = policy.preference_gradient(logits, actions, offsets, ref, **k)
    want = O.preference(logits, actions, offsets, ref, **k)
    dtype = logits.dtype
    assert got.dlogits.dtype == dtype
    for name, t in (("stats", got.stats), ("ratios", got.ratios), ("dlogits", got.dlogits)):
        v, b = want[name]
        t = t.cpu().double()
        dt = dtype if name == "dlogits" else torch.float32
        inf = v.isinf()
        assert torch.equal(t[inf], v[inf]), name
        info = torch.finfo(dt)
        limit = b + (v.abs() + b) * info.eps / 2 + info.smallest_normal * info.eps / 2 + 2.0 ** -120
        worst = ((t - v).abs() / limit)[~inf]
        assert not worst.numel() or worst.max() <= 1, f"{name}: {worst.max():.2f} times the bound"
    again = policy.preference_gradient(logits, actions, offsets, ref, **k)
    assert all(torch.equal(a, b) for a, b in zip(got, again) if not a.isnan().any())
    return got


HEADS = [1, 2, 3, 4, 7, 8, 12, 15, 16, 17, 31, 32, 33, 63, 64, 65, 66, 100, 129, 513, 1024, 2049, 4099, 16381]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("A", HEADS)
def test_heads(A, dtype):
    _check(*_inputs([3, 1, 0, 4, 2, 2], A, dtype, seed=A)[:4], beta=0.7)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("A", [32769, 70001])
def test_long_rows(A, dtype):
    _check(*_inputs([2, 1], A, dtype)[:4], beta=0.7)


@pytest.mark.parametrize("A", [5, 12, 40, 200])
@pytest.mark.parametrize("lengths", [[1, 1], [256, 0], [0, 0], [100, 156], [200, 300], [31, 1], [32, 33], [700, 20, 1, 0, 3, 257]])
def test_lengths(lengths, A):
    _check(*_inputs(lengths, A, unused=0.2)[:4], beta=0.3)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("A, pad", [(6, 1), (12, 0), (12, 4), (12, 3), (50, 7), (300, 5), (5000, 1)])
def test_masks_and_rows_apart(A, pad, dtype):
    l, a, o, r, m = _inputs([5, 9, 40, 33], A, dtype, pad=pad, mask=0.5, unused=0.1)
    _check(l, a, o, r, mask=m, beta=0.5)
    first = m[0].clone()
    first[a.clamp(min=0)] = True
    _check(l, a, o, r, mask=first, beta=0.5)                       # one row for all
    wide = torch.zeros(m.shape[0], A + 3, dtype=torch.uint8, device="cuda")[:, 1:A + 1].copy_(m)
    _check(l, a, o, r, mask=wide, beta=0.5)


@pytest.mark.parametrize("A", [12, 64, 1000])
@pytest.mark.parametrize("k", [dict(), dict(smoothing=0.2), dict(average=True, beta=3.0), dict(denominator=7.5), dict(weights=True),
                               dict(weights=True, average=True, smoothing=0.05, beta=2.0), dict(weights=True, denominator=3.0)])
def test_options(A, k):
    l, a, o, r, _ = _inputs([7, 3, 20, 33, 2, 2, 1, 50], A, unused=0.3)
    if "weights" in k:
        k = dict(k, weights=torch.tensor([0.5, 0.0, 2.0, 1.0]).cuda())
    _check(l, a, o, r, **k)
    _check(l, a, o, None, **k)


@pytest.mark.parametrize("pairs", [1, 100, 3000, 5001])
def test_many_pairs(pairs):
    g = torch.Generator().manual_seed(1)
    lengths = torch.randint(0, 4, (2 * pairs,), generator=g).tolist()
    w = torch.rand(pairs, generator=g).cuda()
    for A in (7, 70):
        l, a, o, r, _ = _inputs(lengths, A)
        _check(l, a, o, r, weights=w)


@pytest.mark.parametrize("A", [3, 12, 50])
@pytest.mark.parametrize("longest", [(40, 20001), (399, 20001), (0, 7000)])
def test_one_long_pair_among_many_short_ones(longest, A):
    """Lengths far from their mean: a pair of thousands of rows is one workgroup's where there are pairs enough."""
    g = torch.Generator().manual_seed(A)
    lengths = torch.randint(0, 5, (400,), generator=g).tolist()
    lengths[longest[0]] = longest[1]
    l, a, o, r, _ = _inputs(lengths, A, unused=0.1, outside=5)
    _check(l, a, o, r, weights=torch.rand(200, generator=g).cuda(), average=True, beta=0.5)


@pytest.mark.parametrize("A", [12, 100])
def test_rows_outside_the_sequences(A):
    l, a, o, r, _ = _inputs([4, 9], A, outside=300)
    l[:5], l[-5:] = float("nan"), float("inf")
    got = _check(l.nan_to_num(0.0, 0.0), a, o, r)
    bad = __import__("paper_2607_26005_amd.policy", fromlist=["x"]).preference_gradient(l, a, o, r)
    assert torch.equal(bad.dlogits, got.dlogits) and torch.equal(bad.stats, got.stats)
    assert (got.dlogits[:300] == 0).all() and (got.dlogits[-300:] == 0).all()


@pytest.mark.parametrize("A", [5, 64, 300])
def test_rows_that_do_not_count(A):
    from paper_2607_26005_amd import policy
    l, a, o, r, _ = _inputs([6, 6], A)
    m = torch.ones(12, A, dtype=torch.bool, device="cuda")
    m[2] = False                                       # nothing allowed
    l[3] = float("nan")
    a[3] = -1                                          # an action of none: not looked at
    a[4] = A                                           # nor one beyond the head
    l[7, 1], m[7, 1] = float("nan"), False             # nor what is masked
    l[8] = -math.inf
    a[7] = 0
    m[7, 0] = True
    r[3] = float("nan")
    got = policy.preference_gradient(l, a, o, r, mask=m, average=True)
    assert got.stats.isfinite().all() and (got.dlogits[[2, 3, 4, 8]] == 0).all() and got.dlogits[7, 1] == 0
    clean, ref = l.clone(), r.clone()
    clean[3], clean[7, 1], ref[3] = 0.0, 0.0, 0.0
    _check(clean, a, o, ref, mask=m, average=True)
    assert torch.equal(policy.preference_gradient(clean, a, o, ref, mask=m, average=True).dlogits, got.dlogits)


@pytest.mark.parametrize("A", [5, 64, 300])
def test_actions_of_probability_zero(A):
    l, a, o, r, _ = _inputs([2, 3, 4, 1], A)
    l[0, 0], a[0] = -math.inf, 0                       # the preferred one could not have been taken
    got = _check(l, a, o, r)
    assert got.stats[0] == math.inf and got.dlogits.isfinite().all() and got.dlogits[0, 0] == 0
    l[3, 1], a[3] = -math.inf, 1                       # nor the other
    from paper_2607_26005_amd import policy
    got = policy.preference_gradient(l, a, o, r)
    assert got.stats[0].isnan() and got.dlogits[:5].isnan().any(1).all() and got.dlogits[5:].isfinite().all()
    w = torch.tensor([0.0, 1.0]).cuda()                # unless that pair is left out
    got = policy.preference_gradient(l, a, o, r, weights=w)
    assert got.stats.isfinite().all() and (got.dlogits[:5] == 0).all() and (got.dlogits[5:] != 0).any()


@pytest.mark.parametrize("A", [5, 64, 300])
def test_no_numbers_stay_in_their_pair(A):
    from paper_2607_26005_amd import policy
    for bad in (float("nan"), float("inf")):
        l, a, o, r, _ = _inputs([2, 3, 4, 1], A)
        l[1, 2] = bad
        got = policy.preference_gradient(l, a, o, r)
        assert got.stats[0].isnan() and got.dlogits[:5].isnan().any(1).all() and got.dlogits[5:].isfinite().all()
        assert got.ratios[0].isnan() and got.ratios[1:].isfinite().all()


def test_extreme_logits_and_margins():
    for A in (12, 300):
        l, a, o, r, _ = _inputs([2, 3, 4, 1], A)
        _check(l * 1e4, a, o, r)
        _check(l * 1e-30, a, o, r)
        _check(l, a, o, r, beta=1e4)
        _check(l, a, o, r * 100, beta=50.0, smoothing=0.1)


def test_nothing_to_learn_from():
    from paper_2607_26005_amd import policy
    for A in (12, 300):
        l, a, o, r, _ = _inputs([2, 3], A)
        got = policy.preference_gradient(l, a, o, r, weights=torch.zeros(1).cuda())
        assert (got.stats == 0).all() and (got.dlogits == 0).all()
        got = policy.preference_gradient(l, a, o[:1], r)
        assert (got.stats == 0).all() and (got.dlogits == 0).all() and got.ratios.shape == (0,)
        got = policy.preference_gradient(l[:0], a[:0], torch.zeros(5, dtype=torch.int64, device="cuda"), r[:0])
        assert got.dlogits.shape == (0, A) and (got.ratios == 0).all()
        assert abs(got.stats[0].item() - math.log(2)) < 1e-6
        got = policy.preference_gradient(l, torch.full_like(a, -1), o, r)
        assert (got.dlogits == 0).all() and abs(got.stats[0].item() - math.log(2)) < 1e-6


def test_offsets_out_of_range_are_cut():
    from paper_2607_26005_amd import policy
    for A in (12, 300):
        l, a, o, r, _ = _inputs([2, 3], A)
        far = torch.tensor([-(1 << 40), 2, 1 << 40]).cuda()
        got, want = policy.preference_gradient(l, a, far, r), policy.preference_gradient(l, a, o, r)
        assert all(map(torch.equal, got, want))


def test_gradient_is_that_of_the_loss():
    from paper_2607_26005_amd import policy
    for A in (11, 90):
        l, a, o, r, _ = _inputs([5, 8, 1, 2], A)
        want, dl = O.by_autograd(l, a, o, r, 0.4)
        got = policy.preference_gradient(l, a, o, r, beta=0.4)
        assert abs(got.stats[0].item() - want) < 1e-5 and torch.allclose(got.dlogits.cpu().double(), dl, rtol=1e-4, atol=1e-7)
        # and against differences of the loss, fp32 off by 1e-7 of about 1 over the step
        d = torch.randn(l.shape, generator=torch.Generator().manual_seed(5)).cuda()
        f = lambda x: policy.preference_gradient(x, a, o, r, beta=0.4).stats[0].double()
        diff = (f(l + 0.01 * d) - f(l - 0.01 * d)) / 0.02
        assert abs(diff - (got.dlogits.double() * d).sum()) < 1e-4 + 2e-3 * abs(diff)


def test_autograd_and_loss_scales():
    from paper_2607_26005_amd import policy
    for dtype in DTYPES:
        l, a, o, r, _ = _inputs([50, 80, 10, 20], 30, dtype)
        x = l.clone().requires_grad_()
        loss, stats, ratios = policy.preference_loss(x, a, o, r, beta=0.1)
        assert loss == stats[0] and not stats.requires_grad and not ratios.requires_grad
        (loss * 4096.0).backward()
        exact, bound = O.preference(l, a, o, r, beta=0.1)["dlogits"]
        exact, bound = exact * 4096, bound * 4096 + 2 * O.U * (exact * 4096).abs()
        info = torch.finfo(dtype)
        # (bfloat16: rounded before the factor, a power of two that changes nothing, and once more)
        limit = bound + (exact.abs() + bound) * info.eps + info.smallest_normal * info.eps
        assert x.grad.dtype == dtype and ((x.grad.cpu().double() - exact).abs() <= limit).all()


def test_parts_add_up():
    from paper_2607_26005_amd import policy
    l, a, o, r, _ = _inputs([5, 8, 1, 2, 7, 7], 20)
    whole = policy.preference_gradient(l, a, o, r, denominator=3.0)
    n = int(o[2])
    one = policy.preference_gradient(l[:n], a[:n], o[:3], r[:n], denominator=3.0)
    two = policy.preference_gradient(l[n:], a[n:], o[2:] - n, r[n:], denominator=3.0)
    assert torch.equal(torch.cat([one.dlogits, two.dlogits]), whole.dlogits)
    assert torch.allclose(one.stats + two.stats, whole.stats, rtol=1e-6)


def test_streams_and_graphs():
    from paper_2607_26005_amd import policy
    w = torch.rand(3000, generator=torch.Generator().manual_seed(2)).cuda()
    for lengths, A, k in (([40, 60, 3, 9], 12, {}), ([40, 60, 3, 9], 700, {}), ([1, 2] * 3000, 12, dict(weights=w))):
        l, a, o, r, _ = _inputs(lengths, A)
        want = policy.preference_gradient(l, a, o, r, **k)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            got = policy.preference_gradient(l, a, o, r, **k)
        torch.cuda.current_stream().wait_stream(side)
        assert all(map(torch.equal, got, want))
        graphs = []
        for _ in range(2):
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                held = policy.preference_gradient(l, a, o, r, **k)
            graphs.append((graph, held))
        for i in range(3):
            l.mul_(0.9)
            want = policy.preference_gradient(l, a, o, r, **k)
            for graph, held in graphs:
                held.dlogits.zero_()
                graph.replay()
                assert all(map(torch.equal, held, want))


def test_rows_beyond_32_bits():
    from paper_2607_26005_amd import policy
    far = 1 << 32
    for A in (12, 90):
        l, a, o, r, _ = _inputs([1, 1], A, torch.bfloat16)
        base = torch.empty(far + 4096, dtype=torch.bfloat16, device="cuda")
        view = torch.as_strided(base, (2, A), (far, 1))
        view.copy_(l)
        got, want = policy.preference_gradient(view, a, o, r), policy.preference_gradient(l, a, o, r)
        assert all(map(torch.equal, got, want))
        del base, view


@pytest.mark.parametrize("A, dtype", [(3, torch.float32), (12, torch.bfloat16), (50, torch.float16), (100, torch.float32)])
def test_long_sequences(A, dtype):
    l, a, o, r, m = _inputs([9000, 3000], A, dtype, mask=0.7, unused=0.1, outside=50)
    got = _check(l, a, o, r, mask=m, beta=0.02)
    assert (got.dlogits[:50] == 0).all() and (got.dlogits[-50:] == 0).all()
    _check(l, a, o, r, mask=m, average=True, weights=torch.tensor([2.0]).cuda(), denominator=3.0)
