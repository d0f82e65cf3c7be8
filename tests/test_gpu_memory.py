"""The gated recurrence on the device against its 64-bit form, step by step on the host:
values, states and gradients within running error bounds (tests/memory_oracle.py)."""
import pytest
import torch

from tests import memory_oracle as O

pytestmark = pytest.mark.gpu

DTYPES = [torch.float32, torch.bfloat16, torch.float16]


@pytest.fixture(autouse=True)
def device():
    if not torch.cuda.is_available():
        pytest.skip("no HIP device")


def _rand(seed, *shape, scale=1.0, shift=0.0):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed)) * scale + shift


def _inputs(B, T, C, dtype, order="batch", resets=0.0, state=True, seed=0, keep=2.0):
    """gates, inputs, state, resets on the device, laid out as asked."""
    g, x = _rand(seed, B, T, C, scale=2.0, shift=keep), _rand(seed + 1, B, T, C)
    r = torch.rand(B, T, generator=torch.Generator().manual_seed(seed + 2)) < resets if resets else None
    if order == "time":
        g, x = (t.transpose(0, 1).contiguous().to("cuda", dtype).transpose(0, 1) for t in (g, x))
        r = None if r is None else r.t().contiguous().cuda().t()
    elif order == "halves":
        both = torch.cat([g, x], 2).to("cuda", dtype)
        g, x = both[..., :C], both[..., C:]
    elif order == "odd":   # rows at an odd distance, off any alignment
        g, x = (torch.zeros(B, T, 2 * C + 3, dtype=dtype, device="cuda")[..., 1:C + 1].copy_(t) for t in (g, x))
    else:
        g, x = g.to("cuda", dtype), x.to("cuda", dtype)
    if r is not None:
        r = r.cuda()
    return g, x, (_rand(seed + 3, B, C).cuda() if state else None), r


def _close(got, want, bound, dtype, what):
    got = got.detach().cpu().double()
    assert got.shape == want.shape, what
    limit = bound + (O.half_step(want.abs() + bound, dtype) if dtype != torch.float32 else O.U * (want.abs() + bound)) + 2.0 ** -126
    worst = ((got - want).abs() / limit).max() if got.numel() else torch.zeros(())
    assert worst <= 1, f"{what}: {worst:.2f} times the bound"


def _check(g, x, s, r, dout=None, dlast=None, grads=True):
    from paper_2607_26005_amd import memory
    dtype = x.dtype
    h, last, eh, el = O.scan(g, x, s, r)
    out, after = memory.gated_scan(g, x, s, r)
    assert out.dtype == dtype and after.dtype == torch.float32
    _close(out, h, eh, dtype, "out")
    _close(after, last, el, torch.float32, "last state")
    if not grads:
        return
    leaves = [t.detach().requires_grad_() for t in (g, x)] + ([] if s is None else [s.detach().requires_grad_()])
    out2, after2 = memory.gated_scan(leaves[0], leaves[1], leaves[2] if s is not None else None, r)
    assert torch.equal(out2, out) and torch.equal(after2, after)   # (saving states changes nothing)
    dout = _rand(7, *x.shape).to("cuda", dtype) if dout is None else dout
    dlast = _rand(8, *after.shape).cuda() if dlast is None else dlast
    got = torch.autograd.grad((out2, after2), leaves, (dout, dlast))
    want, bounds = O.scan_gradient(g, x, s, r, dout, dlast)
    for name, a, w, b, dt in zip(("dgates", "dinputs", "dstate"), got, want, bounds, (dtype, dtype, torch.float32)):
        assert a.dtype == dt
        _close(a, w, b, dt, name)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("B, T, C", [(1, 1, 1), (3, 1, 7), (2, 2, 64), (5, 15, 12), (4, 16, 33), (2, 17, 128), (1, 47, 5),
                                     (7, 64, 10), (2, 127, 66), (1, 128, 300)])
def test_small_sequences(B, T, C, dtype):
    _check(*_inputs(B, T, C, dtype, resets=0.1))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("order", ["batch", "time", "halves", "odd"])
@pytest.mark.parametrize("state", [True, False])
def test_layouts(order, dtype, state):
    _check(*_inputs(3, 37, 34, dtype, order=order, resets=0.2, state=state))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("B, T, C, resets", [(1, 128, 2, 0.0), (1, 131, 3, 0.05), (2, 1000, 6, 0.0), (1, 2049, 64, 0.002),
                                             (1, 4113, 10, 0.0), (3, 777, 130, 0.01)])
def test_steps_cut_into_segments(B, T, C, resets, dtype):
    _check(*_inputs(B, T, C, dtype, resets=resets, keep=4.0))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("B, T, C, order", [(1, 1500, 7, "batch"), (2, 700, 131, "odd"), (3, 515, 129, "time"), (1, 600, 1, "batch")])
def test_tiles_of_odd_channels(B, T, C, order, dtype):
    _check(*_inputs(B, T, C, dtype, order=order, resets=0.003, keep=4.0))


def test_one_long_sequence_of_few_channels():
    # 512 segments in 32 groups
    _check(*_inputs(1, 40003, 2, torch.float32, resets=0.0005, keep=7.0))


def test_segments_with_state_kept_through():
    # gates that keep nearly everything: the first state is still there at the end
    g, x, s, r = _inputs(1, 3000, 8, torch.float32, keep=14.0)
    _check(g, x, s * 100, None)


def test_results_do_not_depend_on_the_batch():
    from paper_2607_26005_amd import memory
    g, x, s, r = _inputs(300, 40, 64, torch.bfloat16, resets=0.1)
    all_, last = memory.gated_scan(g, x, s, r)
    for b in (0, 7, 299):
        one, l1 = memory.gated_scan(g[b:b + 1], x[b:b + 1], s[b:b + 1], r[b:b + 1])
        assert torch.equal(one[0], all_[b]) and torch.equal(l1[0], last[b])


def test_a_cut_sequence_goes_on_from_its_state():
    from paper_2607_26005_amd import memory
    g, x, s, _ = _inputs(2, 50, 20, torch.float32)
    whole, last = memory.gated_scan(g, x, s)
    a, mid = memory.gated_scan(g[:, :23], x[:, :23], s)
    b, end = memory.gated_scan(g[:, 23:], x[:, 23:], mid)
    assert torch.equal(torch.cat([a, b], 1), whole) and torch.equal(end, last)


def test_packed_sequences_are_those_alone():
    from paper_2607_26005_amd import memory
    lengths = [1, 30, 7, 64, 2, 200]
    T = sum(lengths)
    g, x, _, _ = _inputs(1, T, 24, torch.float32, state=False)
    resets = torch.zeros(1, T, dtype=torch.bool, device="cuda")
    at = 0
    for n in lengths:
        resets[0, at] = True
        at += n
    out, _ = memory.gated_scan(g, x, None, resets)
    at = 0
    for n in lengths:
        h, _, e, _ = O.scan(g[:, at:at + n], x[:, at:at + n])
        _close(out[:, at:at + n], h, e, torch.float32, f"{n} steps")
        at += n


@pytest.mark.parametrize("T", [40, 700])
def test_a_reset_forgets_what_is_no_number(T):
    from paper_2607_26005_amd import memory
    g, x, s, _ = _inputs(1, T, 6, torch.float32)
    resets = torch.zeros(1, T, dtype=torch.uint8, device="cuda")
    cut = T // 2 + 3
    resets[0, cut] = 1
    clean, _ = memory.gated_scan(g[:, cut:], x[:, cut:])
    x = x.clone()
    x[0, 5, 0], x[0, 6, 1], s[0, 2] = float("nan"), float("inf"), float("nan")
    leaves = [t.requires_grad_() for t in (g.clone(), x, s)]
    out, last = memory.gated_scan(*leaves, resets)
    assert out[0, 5:cut, 0].isnan().all() and out[0, 6, 1].isinf() and out[0, :cut, 2].isnan().all()
    assert out[0, cut:].isfinite().all() and last.isfinite().all()
    assert torch.allclose(out[0, cut:], clean[0], rtol=1e-5, atol=1e-6)
    dout = torch.zeros_like(out)
    dout[0, cut + 4:] = 1.0
    dg, dx, ds = torch.autograd.grad(out, leaves, dout)
    assert dx[0, cut:].isfinite().all() and (dx[0, :cut] == 0).all() and (ds == 0).all()
    # a gradient that is no number stays on its side as well
    dout[0, cut + 4:] = float("nan")
    dout[0, 3] = 1.0
    out, _ = memory.gated_scan(*leaves, resets)
    _, dx, _ = torch.autograd.grad(out, leaves, dout)
    assert dx[0, cut:cut + 5].isnan().all() and dx[0, :4].isfinite().all() and (dx[0, 4:cut] == 0).all()


def _kind(t):
    """0 of what is finite, 1 and -1 of the infinities, 2 of NaN."""
    t = t.detach().cpu().double()
    return torch.where(t.isnan(), torch.full_like(t, 2.0), torch.where(t.isinf(), t.sign(), torch.zeros_like(t)))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("B, T, C, resets", [(1, 40, 6, 0.0), (1, 1500, 6, 0.0), (2, 1500, 5, 0.003), (1, 9000, 2, 0.0)])
def test_infinities_stay_as_the_formula_has_them(B, T, C, resets, dtype):
    """An infinite state remains one until a reset, however many steps lie behind and however they
    are cut: the product of their gates is below fp32's range, and not 0."""
    from paper_2607_26005_amd import memory
    inf = float("inf")
    g, x, s, r = _inputs(B, T, C, dtype, resets=resets, keep=0.0)
    x[0, 9, 0], x[0, 11, 1] = inf, -inf
    x[0, T // 2, 1] = inf    # against the one before: no number from here on
    x[-1, T - 20, -1] = -inf
    s[0, 0] = -inf           # against step 9's
    if B > 1:
        s[1, 1] = inf
    want, last, *_ = O.scan(g, x, s, r)
    out, after = memory.gated_scan(g, x, s, r)
    assert torch.equal(_kind(out), _kind(want)) and torch.equal(_kind(after), _kind(last))
    assert (_kind(want) == 1).any() or resets == 0.0
    # and backwards
    g, x, s, _ = _inputs(B, T, C, dtype, seed=5, keep=0.0)
    dout, dlast = _rand(7, B, T, C).to("cuda", dtype), _rand(8, B, C).cuda()
    dout[0, T - 9, 0], dout[0, T - 11, 1], dout[0, T // 2, 1], dlast[0, 0] = inf, -inf, inf, -inf
    leaves = [t.requires_grad_() for t in (g, x, s)]
    got = torch.autograd.grad(memory.gated_scan(*leaves, r), leaves, (dout, dlast))
    grads, _ = O.scan_gradient(g, x, s, r, dout, dlast)
    for name, a, w in zip(("dgates", "dinputs", "dstate"), got, grads):
        assert torch.equal(_kind(a), _kind(w)), name


def test_gates_at_their_ends():
    from paper_2607_26005_amd import memory
    inf = float("inf")
    gates = torch.tensor([-inf, -200.0, -90.0, -20.0, 0.0, 20.0, 90.0, 200.0, inf, float("nan")]).cuda()
    g = gates.view(1, 1, -1).clone()
    x, s = torch.full_like(g, 3.0), torch.full_like(g[0], 5.0)
    out, _ = memory.gated_scan(g, x, s)
    want = 5 * gates.double().sigmoid() + 3 * (-gates.double()).sigmoid()
    assert torch.allclose(out[0, 0, :-1].double(), want[:-1], rtol=2e-6, atol=0) and out[0, 0, -1].isnan()
    leaves = [t.requires_grad_() for t in (g, x, s)]
    out, _ = memory.gated_scan(*leaves)
    dg, dx, ds = torch.autograd.grad(out, leaves, torch.ones_like(out))
    ends = [0, 1, 7, 8]
    assert (dg[0, 0, ends] == 0).all() and dx[0, 0, :2].tolist() == [1.0, 1.0] and ds[0, 7:9].tolist() == [1.0, 1.0]
    # small parts keep their own precision
    b = (-gates[3:7].double()).sigmoid()
    assert torch.allclose(dx[0, 0, 3:6].double(), b[:3], rtol=1e-6, atol=0)


def test_gradients_against_differences():
    from paper_2607_26005_amd import memory
    g, x, s, r = (t if t is None else t.requires_grad_(t.is_floating_point()) for t in
                  _inputs(2, 21, 5, torch.float32, resets=0.1))
    w, wl = _rand(11, 2, 21, 5).cuda(), _rand(12, 2, 5).cuda()

    def loss(g, x, s):
        out, last = memory.gated_scan(g, x, s, r)
        return (out.double() * w).sum() + (last.double() * wl).sum()

    grads = torch.autograd.grad(loss(g, x, s), (g, x, s))
    gen = torch.Generator().manual_seed(3)
    for k, t in enumerate((g, x, s)):
        d = torch.randn(t.shape, generator=gen).cuda()
        step = 1e-2
        args = [g, x, s]
        with torch.no_grad():
            ends = []
            for sign in (1, -1):
                moved = list(args)
                moved[k] = t + sign * step * d
                ends.append(loss(*moved))
        # a central difference: step^2 / 6 of a third derivative (below some 1e-4 of the sum here), and
        # fp32 values of about 1 in 400 terms, over the step
        got, want = (grads[k].double() * d).sum(), (ends[0] - ends[1]) / (2 * step)
        assert abs(got - want) <= 2e-3 * (grads[k].double() * d).abs().sum(), (k, got, want)


def test_gradients_that_arrive_in_other_forms():
    from paper_2607_26005_amd import memory
    g, x, s, r = _inputs(2, 33, 6, torch.float32, resets=0.1)
    leaves = [t.requires_grad_() for t in (g, x, s)]
    one, last1 = torch.ones(2, 33, 6, device="cuda"), torch.ones(2, 6, device="cuda")
    run = lambda: memory.gated_scan(*leaves, r)
    want = torch.autograd.grad(run()[0], leaves, one)
    assert all(map(torch.equal, torch.autograd.grad(run()[0].sum(), leaves), want))          # expanded
    got = torch.autograd.grad(run()[0].permute(2, 0, 1).contiguous(), leaves, one.permute(2, 0, 1).contiguous())
    assert all(map(torch.equal, got, want))                                                    # channels outermost
    last_only = torch.autograd.grad(run()[1].sum(), leaves)
    zero = torch.zeros_like(one)
    assert all(map(torch.equal, last_only, torch.autograd.grad(run(), leaves, (zero, last1))))
    assert torch.equal(torch.autograd.grad(run()[0].sum(), leaves[1])[0], want[1])             # some of them alone
    x2 = torch.zeros(1, 1, 6, device="cuda", requires_grad=True)                               # one input for all steps
    got, = torch.autograd.grad(memory.gated_scan(leaves[0], x2.expand(2, 33, 6), leaves[2], r)[0].sum(), x2)
    x3 = x2.detach().expand(2, 33, 6).contiguous().requires_grad_()
    each, = torch.autograd.grad(memory.gated_scan(leaves[0], x3, leaves[2], r)[0].sum(), x3)
    assert torch.allclose(got[0, 0], each.sum((0, 1)), rtol=1e-5)


def test_nothing_to_do():
    from paper_2607_26005_amd import memory
    z = lambda *s: torch.zeros(*s, device="cuda", requires_grad=True)
    out, last = memory.gated_scan(z(0, 5, 4), z(0, 5, 4))
    assert out.shape == (0, 5, 4) and last.shape == (0, 4)
    s = torch.randn(3, 4, device="cuda", requires_grad=True)
    g, x = z(3, 0, 4), z(3, 0, 4)
    out, last = memory.gated_scan(g, x, s)
    assert out.shape == (3, 0, 4) and torch.equal(last, s)
    ds, = torch.autograd.grad((last * 2).sum(), s)
    assert (ds == 2).all()
    assert memory.gated_step(z(0, 4).detach(), z(0, 4).detach(), torch.zeros(0, 4, device="cuda")).shape == (0, 4)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("given", [True, False])
def test_the_gradient_of_no_steps(given, dtype):
    """A rollout of no steps has gradients too, whether or not its state wants one."""
    from paper_2607_26005_amd import memory
    g, x = (torch.zeros(3, 0, 4, device="cuda", dtype=dtype, requires_grad=True) for _ in range(2))
    s = torch.randn(3, 4, device="cuda") if given else None
    out, last = memory.gated_scan(g, x, s)
    assert out.shape == (3, 0, 4) and torch.equal(last, s if given else torch.zeros_like(last))
    dg, dx = torch.autograd.grad(out.sum() + (last * 2).sum(), (g, x))
    assert dg.shape == dx.shape == (3, 0, 4) and dg.dtype == dx.dtype == dtype


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("B, C", [(1, 1), (5, 7), (8, 128), (300, 40), (3, 513)])
def test_single_steps_are_the_scan(B, C, dtype):
    from paper_2607_26005_amd import memory
    for order in ("batch", "halves", "odd"):
        g, x, s, r = _inputs(B, 4, C, dtype, order=order, resets=0.2)
        out, last = memory.gated_scan(g, x, s, r)
        state = s.clone()
        v = state._version
        for t in range(4):
            y = memory.gated_step(g[:, t], x[:, t], state, r[:, t])
            assert torch.equal(y, out[:, t]), (order, t)
        assert torch.equal(state, last) and state._version == v + 4
        # in place of the inputs, without resets
        a, b = x[:, 0].clone(), s.clone()
        want = memory.gated_step(g[:, 0], a, b.clone())
        assert memory.gated_step(g[:, 0], a, b, out=a) is a and torch.equal(a, want)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("B, C", [(1, 1), (5, 7), (300, 40), (3, 513), (64, 2050)])
def test_a_step_in_place(B, C, dtype):
    """What a step writes may be its own operands' memory."""
    from paper_2607_26005_amd import memory
    g, x, s, r = (t[:, 0] if t.dim() == 3 else t for t in _inputs(B, 1, C, dtype, resets=0.3))
    r = r[:, 0]
    held = s.clone()
    want = memory.gated_step(g, x, held, r)
    both = torch.cat([g, x, torch.zeros_like(g)], 1)
    for k in range(3):   # over the gates, over the inputs, between them
        rows, state = both.clone(), s.clone()
        got = memory.gated_step(rows[:, :C], rows[:, C:2 * C], state, r, rows[:, k * C:(k + 1) * C])
        assert torch.equal(got, want) and torch.equal(state, held)
        left = [i for i in range(3) if i != k]
        assert all(torch.equal(rows[:, i * C:(i + 1) * C], both[:, i * C:(i + 1) * C]) for i in left)
    if dtype == torch.float32:
        state = s.clone()
        assert memory.gated_step(g, x, state, r, state) is state and torch.equal(state, held)
        state = x.clone()   # the inputs are the state
        want = memory.gated_step(g, x, x.clone(), r)
        assert torch.equal(memory.gated_step(g, state, state, r), want) and torch.equal(state, want)


def test_rows_and_channels_beyond_are_left():
    from paper_2607_26005_amd import memory, pictura
    g, x, s, _ = _inputs(2, 20, 6, torch.float32)
    held = torch.full((2, 24, 9), 7.0, device="cuda")
    pictura.pictura_gated_scan(g, x, held[:, 2:22, 1:7], torch.empty_like(s), state=s)
    out, _ = memory.gated_scan(g, x, s)
    assert torch.equal(held[:, 2:22, 1:7], out)
    held[:, 2:22, 1:7] = 7.0
    assert (held == 7.0).all()


def test_other_streams_and_graphs():
    from paper_2607_26005_amd import memory
    g, x, s, r = _inputs(2, 700, 32, torch.bfloat16, resets=0.01)
    want, last = memory.gated_scan(g, x, s, r)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got, _ = memory.gated_scan(g, x, s, r)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got, want)
    graphs = []
    for _ in range(2):   # two graphs, replayed in turn
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = memory.gated_scan(g, x, s, r)
        graphs.append((graph, out))
    state, y = s.clone(), None
    step = torch.cuda.CUDAGraph()
    with torch.cuda.graph(step):
        y = memory.gated_step(g[:, 0], x[:, 0], state)
    for k in range(3):
        x.copy_(_rand(50 + k, *x.shape))
        want, last = memory.gated_scan(g, x, s, r)
        for graph, out in graphs:
            out[0].zero_()
            graph.replay()
            assert torch.equal(out[0], want) and torch.equal(out[1], last)
        now = state.clone()
        step.replay()
        assert torch.equal(memory.gated_step(g[:, 0], x[:, 0], now), y) and torch.equal(now, state)


def test_gradient_in_a_graph():
    from paper_2607_26005_amd import pictura
    g, x, s, r = _inputs(3, 300, 10, torch.float32, resets=0.02)
    out, last = torch.empty_like(x), torch.empty_like(s)
    saved = torch.empty(-(-300 // pictura.SCAN_STEPS), 3, 10, device="cuda")
    dout, dlast = _rand(4, 3, 300, 10).cuda(), _rand(5, 3, 10).cuda()
    grads = [torch.empty_like(t) for t in (g, x, s)]

    def both():
        pictura.pictura_gated_scan(g, x, out, last, saved, s, r)
        pictura.pictura_gated_scan_gradient(g, x, saved, dout, dlast, *grads, r)

    both()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    for k in range(3):
        x.copy_(_rand(60 + k, *x.shape))
        both()
        want = [t.clone() for t in grads]
        for t in grads:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(map(torch.equal, grads, want))


def test_offsets_beyond_32_bits():
    # 2^32 elements between the two sequences' tensors, only some of them touched
    from paper_2607_26005_amd import memory
    far = 1 << 32
    base = torch.empty(far + 4096, dtype=torch.bfloat16, device="cuda")
    g, x, s, _ = _inputs(2, 20, 64, torch.bfloat16)
    view = torch.as_strided(base, (2, 20, 64), (far, 128, 1))
    view.copy_(x)
    g2 = torch.as_strided(base, (2, 20, 64), (far, 128, 1), 64)
    g2.copy_(g)
    want, last = memory.gated_scan(g, x, s)
    got, last2 = memory.gated_scan(g2, view, s)
    assert torch.equal(got, want) and torch.equal(last, last2)


def test_padding_behind_a_reset_may_hold_anything():
    from paper_2607_26005_amd import memory
    for T, n in ((30, 17), (900, 500)):
        g, x, s, _ = _inputs(1, T, 6, torch.float32)
        resets = torch.zeros(1, T, dtype=torch.bool, device="cuda")
        resets[0, n] = True
        leaves = [t.clone().requires_grad_() for t in (g[:, :n], x[:, :n], s)]
        out, _ = memory.gated_scan(*leaves)
        dout = _rand(3, 1, n, 6).cuda()
        want = torch.autograd.grad(out, leaves, dout)
        with torch.no_grad():
            g[:, n:], x[:, n:] = float("nan"), float("inf")
        padded = [t.clone().requires_grad_() for t in (g, x, s)]
        got, _ = memory.gated_scan(*padded, resets)
        # (cut into tiles or not: the same to a few units)
        assert torch.allclose(got[:, :n], out, rtol=1e-5, atol=1e-6)
        grads = torch.autograd.grad(got, padded, torch.cat([dout, torch.zeros(1, T - n, 6, device="cuda")], 1))
        for a, b in zip(grads[:2], want[:2]):
            assert torch.allclose(a[:, :n], b, rtol=1e-4, atol=1e-6)
        assert torch.allclose(grads[2], want[2], rtol=1e-4, atol=1e-6)


def test_gradients_are_not_differentiated_again():
    from paper_2607_26005_amd import memory, policy
    g, x, s, _ = _inputs(2, 9, 4, torch.float32)
    x.requires_grad_()
    w = torch.ones(4, device="cuda", requires_grad=True)
    l = torch.randn(4, 5, device="cuda", requires_grad=True)
    a, o = torch.zeros(4, dtype=torch.int64, device="cuda"), torch.tensor([0, 2, 4]).cuda()
    for f, t in ((lambda: memory.gated_scan(g, x, s)[0], x), (lambda: memory.rms_norm(x, w), x),
                 (lambda: memory.rms_norm(x, w, x.detach())[0], x), (lambda: policy.preference_loss(l, a, o)[0], l)):
        once, = torch.autograd.grad(f().sum(), t, create_graph=True)
        plain, = torch.autograd.grad(f().sum(), t)
        assert torch.equal(once, plain)
        with pytest.raises(RuntimeError, match="differentiate twice"):
            once.pow(2).sum().backward()
        if t is not l:   # (that loss does not keep its logits: they are told to be unused)
            once, = torch.autograd.grad(f().sum(), t, create_graph=True)
            with pytest.raises(RuntimeError, match="differentiate twice"):
                torch.autograd.grad(once.pow(2).sum() + t.sum(), t)


def test_a_graph_can_be_gone_through_again():
    from paper_2607_26005_amd import memory
    g, x, s, r = _inputs(2, 600, 4, torch.float32, resets=0.01)
    x.requires_grad_()
    out, _ = memory.gated_scan(g, x, s, r)
    a, = torch.autograd.grad(out.sum(), x, retain_graph=True)
    b, = torch.autograd.grad(out.sum(), x)
    assert torch.equal(a, b)
    with torch.no_grad():
        x.add_(1)
    out, _ = memory.gated_scan(g, x, s, r)
    with torch.no_grad():
        x.add_(1)
    with pytest.raises(RuntimeError, match="modified by an inplace"):
        out.sum().backward()


def test_a_capture_refuses_leaves_that_an_eager_graph_holds():
    from paper_2607_26005_amd import memory, pictura
    x, w = torch.randn(6, 16, device="cuda"), torch.ones(16, device="cuda", requires_grad=True)
    held = w * 1   # an eager graph of the leaf, on the default stream
    memory.rms_norm(x, w)
    graph = torch.cuda.CUDAGraph()
    with pytest.raises(pictura.PicturaError, match="weight: a graph recorded on another stream"):
        with torch.cuda.graph(graph):
            memory.rms_norm(x, w)
    del held
    torch.cuda.synchronize()
    # without one the backward is captured
    graph = torch.cuda.CUDAGraph()
    dy = torch.randn_like(x)
    with torch.cuda.graph(graph):
        dw, = torch.autograd.grad(memory.rms_norm(x, w), w, dy)
    for _ in range(3):
        x.copy_(torch.randn_like(x))
        dw.zero_()
        graph.replay()
        want, = torch.autograd.grad(memory.rms_norm(x, w), w, dy)
        assert torch.equal(dw, want)


def test_gradients_with_a_tangent_or_not_seen():
    """What arrives in the backward is looked at as what goes in."""
    import torch.autograd.forward_ad as forward_ad
    from torch.utils._python_dispatch import TorchDispatchMode
    from paper_2607_26005_amd import memory

    class Mode(TorchDispatchMode):
        def __torch_dispatch__(self, func, types, args=(), kwargs=None):
            return func(*args, **(kwargs or {}))

    g, x, s, r = _inputs(2, 9, 4, torch.float32, resets=0.1)
    x.requires_grad_()
    w = torch.ones(4, device="cuda")
    for f, name in ((lambda: memory.gated_scan(g, x, s, r)[0], "gated_scan"), (lambda: memory.rms_norm(x, w), "rms_norm"),
                    (lambda: memory.rms_norm(x, w, x.detach())[0], "rms_norm")):
        y = f()
        with forward_ad.dual_level():
            dy = forward_ad.make_dual(torch.ones_like(y), torch.ones_like(y))
            with pytest.raises(RuntimeError, match="has a tangent"):
                torch.autograd.grad(y, x, dy, retain_graph=True)
        dy = torch.ones_like(y)
        with Mode(), pytest.raises(RuntimeError, match=f"gradient of {name}: called under a dispatch mode"):
            torch.autograd.grad(y, x, dy, retain_graph=True)
        assert torch.equal(torch.autograd.grad(y, x, dy)[0], torch.autograd.grad(f(), x, dy)[0])
