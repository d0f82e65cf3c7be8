"""The root-mean-square norm on the device against its 64-bit form on the host
(tests/memory_oracle.py): rows, gradients, 8-bit codes to the bit."""
import pytest
import torch

from tests import memory_oracle as O

pytestmark = pytest.mark.gpu

DTYPES = [torch.float32, torch.bfloat16, torch.float16]
WIDTHS = [1, 2, 3, 5, 8, 9, 31, 64, 65, 100, 128, 129, 256, 300, 512, 513, 1000, 1024, 2047, 4096, 5001, 8192, 9001, 16384]


@pytest.fixture(autouse=True)
def device():
    if not torch.cuda.is_available():
        pytest.skip("no HIP device")


def _rand(seed, *shape, scale=1.0, shift=0.0):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed)) * scale + shift


def _rows(seed, n, c, dtype, pad=0, scale=1.0):
    """Rows pad + c elements apart, off any alignment where pad is odd."""
    t = torch.zeros(n, c + pad, dtype=dtype, device="cuda")[:, pad // 2:pad // 2 + c]
    return t.copy_(_rand(seed, n, c, scale=scale))


def _close(got, want, bound, dtype, what):
    got = got.detach().cpu().double()
    limit = bound + O.half_step(want.abs() + bound, dtype) + 2.0 ** -126
    assert got.shape == want.shape, what
    worst = ((got - want).abs() / limit).max() if got.numel() else torch.zeros(())
    assert worst <= 1, f"{what}: {worst:.2f} times the bound"


def _check(n, c, dtype, weight_dtype=torch.float32, residual=True, pad=0, eps=1e-6, scale=1.0):
    from paper_2607_26005_amd import memory
    x, w = _rows(1, n, c, dtype, pad, scale), _rand(2, c, scale=0.3, shift=1.0).to("cuda", weight_dtype)
    r = _rows(3, n, c, dtype, 2 * pad, 2 * scale) if residual else None
    s, y, q = O.norm(x, w, r, eps)
    got = memory.rms_norm(x, w, r, eps)
    out, total = got if residual else (got, None)
    assert out.dtype == dtype
    _close(out, y, 4 * O.U * y.abs(), dtype, "out")
    if residual:
        assert torch.equal(total.cpu(), s)
    leaves = [t.detach().requires_grad_() for t in ((x, w, r) if residual else (x, w))]
    got = memory.rms_norm(leaves[0], leaves[1], leaves[2] if residual else None, eps)
    assert torch.equal(got[0] if residual else got, out)
    dy, ds = _rows(4, n, c, dtype, pad), _rows(5, n, c, dtype) if residual else None
    grads = torch.autograd.grad(got, leaves, (dy, ds) if residual else dy)
    (dx, dw), (bx, bw) = O.norm_gradient(s, w, eps, dy, ds)
    _close(grads[0], dx, bx, dtype, "dx")
    _close(grads[1], dw, bw, weight_dtype, "dweight")
    if residual:
        assert torch.equal(grads[2], grads[0])


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("width", WIDTHS)
def test_widths(width, dtype):
    _check(7, width, dtype, residual=width % 2 == 0)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("width", [16390, 32768, 40001, 65536])
def test_the_widest_rows(width, dtype):
    _check(3, width, dtype)


@pytest.mark.parametrize("rows, width", [(1, 512), (2, 8), (33, 100), (1000, 24), (5000, 136), (3001, 515), (700, 4100)])
@pytest.mark.parametrize("dtype", DTYPES)
def test_many_rows(rows, width, dtype):
    _check(rows, width, dtype)


@pytest.mark.parametrize("dtype", DTYPES[1:])
@pytest.mark.parametrize("width", [6, 40, 512, 3001])
def test_weights_of_the_rows_type(width, dtype):
    _check(9, width, dtype, weight_dtype=dtype)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("pad", [1, 3, 8])
@pytest.mark.parametrize("width", [5, 64, 331, 2050])
def test_rows_apart(width, pad, dtype):
    _check(11, width, dtype, pad=pad)


@pytest.mark.parametrize("scale, eps", [(1e-3, 1e-6), (300.0, 1e-6), (1e-4, 0.0), (1.0, 1.0)])
def test_sizes_of_values(scale, eps):
    for dtype in DTYPES:
        _check(5, 300, dtype, eps=eps, scale=scale)


@pytest.mark.parametrize("kind", [torch.int8, torch.float8_e4m3fn])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows, width, pad", [(1, 1, 0), (3, 7, 1), (65, 64, 0), (40, 333, 3), (300, 512, 0), (20, 4100, 0), (5, 16500, 1),
                                              (2, 65536, 0)])
def test_codes_to_the_bit(rows, width, pad, dtype, kind):
    from paper_2607_26005_amd import memory
    x, w = _rows(1, rows, width, dtype, pad), _rand(2, width, scale=0.3, shift=1.0).cuda()
    for r in (None, _rows(3, rows, width, dtype, pad)):
        held = memory.rms_norm_8bit(x, w, r, dtype=kind)
        codes, scales = O.norm_codes(x, w, r, 1e-6, kind)
        assert held.codes.dtype == kind and held.codes.shape == x.shape
        assert torch.equal(held.scales.cpu(), scales)
        assert torch.equal(held.codes.cpu().view(torch.uint8), codes.view(torch.uint8))
        assert (held.sum is None) == (r is None)
        if r is not None:
            assert torch.equal(held.sum, memory.rms_norm(x, w, r)[1])
        want = codes.float() * scales[:, None]
        assert torch.equal(held.values().cpu(), want)
        out = torch.empty(rows, width, device="cuda")
        assert held.values(out) is out and torch.equal(out.cpu(), want)


def test_every_code_stands_for_its_value():
    from paper_2607_26005_amd import memory
    for kind in (torch.int8, torch.float8_e4m3fn):
        codes = torch.arange(256, dtype=torch.uint8).view(kind)[None].repeat(3, 1).cuda()
        scales = torch.tensor([1.0, 0.37, 2.0 ** -60]).cuda()
        got = memory.RowCodes(codes, scales, None).values().cpu()
        want = codes.cpu().float() * scales.cpu()[:, None]
        assert torch.equal(got.nan_to_num(7), want.nan_to_num(7)) and torch.equal(got.isnan(), want.isnan())


def test_rounding_of_codes():
    # with a weight that makes y what it is told: ties go to the even code
    from paper_2607_26005_amd import memory
    for kind, most in ((torch.int8, 127.0), (torch.float8_e4m3fn, 448.0)):
        y = torch.arange(-2 * int(most), 2 * int(most) + 1).float() / 2
        w = y.cuda()
        x = torch.ones(1, len(y), device="cuda")
        held = memory.rms_norm_8bit(x, w, eps=0.0, dtype=kind)
        assert held.scales.item() == 1.0
        want = y.round() if kind == torch.int8 else y.to(kind).float()
        assert torch.equal(held.values().cpu()[0], want)


def test_rows_that_are_zero_or_no_number():
    from paper_2607_26005_amd import memory
    x = torch.randn(6, 40, device="cuda")
    x[1] = 0.0
    x[2, 7] = float("nan")
    x[3, 8] = float("inf")
    x[4] *= 1e-30
    w = torch.ones(40, device="cuda")
    y = memory.rms_norm(x, w, eps=0.0)
    assert y[[0, 4, 5]].isfinite().all() and torch.allclose(y[4].pow(2).mean(), y.new_ones(()))
    assert y[1].isnan().all() and y[2].isnan().all() and y[3, 8].isnan()   # (0 / 0 without an eps)
    y = memory.rms_norm(x, w)
    assert (y[1] == 0).all()
    for kind in (torch.int8, torch.float8_e4m3fn):
        held = memory.rms_norm_8bit(x, w, dtype=kind)
        v = held.values()
        assert (v[1] == 0).all() and held.scales[1] == 0 and v[2].isnan().all() and v[3].isnan().all()
        assert v[[0, 4, 5]].isfinite().all()
        # an infinity that the norm does not make: a weight's
        w2 = w.clone()
        w2[3] = float("inf")
        assert memory.rms_norm_8bit(x[:1], w2, dtype=kind).values().isnan().all()


def test_results_do_not_depend_on_the_batch():
    from paper_2607_26005_amd import memory
    for c in (24, 512, 5001):
        x, r, w = _rows(1, 600, c, torch.bfloat16), _rows(2, 600, c, torch.bfloat16), _rand(3, c).cuda()
        y, s = memory.rms_norm(x, w, r)
        one, s1 = memory.rms_norm(x[77:78], w, r[77:78])
        assert torch.equal(one[0], y[77]) and torch.equal(s1[0], s[77])


def test_leading_dimensions_and_layouts():
    from paper_2607_26005_amd import memory
    x, r, w = (_rand(k, *s).cuda() for k, s in ((1, (4, 5, 24)), (2, (4, 5, 24)), (3, (24,))))
    y, s = memory.rms_norm(x, w, r)
    flat, sf = memory.rms_norm(x.view(20, 24), w, r.view(20, 24))
    assert y.shape == x.shape and torch.equal(y.view(20, 24), flat) and torch.equal(s.view(20, 24), sf)
    t = lambda a: a.transpose(0, 1).contiguous().transpose(0, 1)
    y2, s2 = memory.rms_norm(t(x), w, t(r))
    assert torch.equal(y2, y) and torch.equal(s2, s)
    assert torch.equal(memory.rms_norm(x.permute(2, 0, 1).contiguous().permute(1, 2, 0), w), memory.rms_norm(x, w))
    assert torch.equal(memory.rms_norm(x[0, 0], w), memory.rms_norm(x, w)[0, 0])
    assert torch.equal(memory.rms_norm(x[0, :1].expand(5, 24), w, r[0])[1], x[0, :1] + r[0])   # one row for all
    held = memory.rms_norm_8bit(x, w, r)
    assert held.codes.shape == x.shape and held.scales.shape == (4, 5) and held.values().shape == x.shape
    leaves = [a.clone().requires_grad_() for a in (x, w, r)]
    y, s = memory.rms_norm(t(leaves[0]), leaves[1], leaves[2])
    got = torch.autograd.grad((y * 2).sum() + s.transpose(0, 1).contiguous().sum(), leaves)
    y, s = memory.rms_norm(leaves[0].view(20, 24), leaves[1], leaves[2].view(20, 24))
    want = torch.autograd.grad((y, s), leaves, (torch.full_like(y, 2.0), torch.ones_like(s)))
    assert all(map(torch.equal, got, want))


def test_gradients_that_are_missing_or_expanded():
    from paper_2607_26005_amd import memory
    x, w, r = (_rand(k, *s).cuda().requires_grad_() for k, s in ((1, (6, 40)), (2, (40,)), (3, (6, 40))))
    y, s = memory.rms_norm(x, w, r)
    dx, dw, dr = torch.autograd.grad(s.sum(), (x, w, r), allow_unused=True)
    assert (dx == 1).all() and (dr == 1).all() and (dw is None or (dw == 0).all())
    y, s = memory.rms_norm(x, w, r)
    a = torch.autograd.grad(y.sum(), (x, w, r))
    y, s = memory.rms_norm(x, w, r)
    b = torch.autograd.grad((y, s), (x, w, r), (torch.ones_like(y), torch.zeros_like(s)))
    assert all(map(torch.equal, a, b))
    y, s = memory.rms_norm(x, w, r)
    assert torch.equal(torch.autograd.grad(y.sum(), w)[0], a[1])
    y, s = memory.rms_norm(x, w, x.detach())   # a residual without a gradient
    assert torch.autograd.grad(y.sum(), x)[0].isfinite().all()
    h = memory.rms_norm(x, w, x)                # the same tensor twice
    dx, = torch.autograd.grad(h[1].sum(), x)
    assert (dx == 2).all()


def test_gradient_against_differences():
    from paper_2607_26005_amd import memory
    x, w, r = (_rand(k, *s).cuda().requires_grad_() for k, s in ((1, (5, 33)), (2, (33,)), (3, (5, 33))))
    a, b = _rand(6, 5, 33).cuda().double(), _rand(7, 5, 33).cuda().double()
    f = lambda *t: sum((o.double() * c).sum() for o, c in zip(memory.rms_norm(*t), (a, b)))
    grads = torch.autograd.grad(f(x, w, r), (x, w, r))
    for k, t in enumerate((x, w, r)):
        d = _rand(20 + k, *t.shape).cuda()
        ends = []
        with torch.no_grad():
            for sign in (1, -1):
                args = [x, w, r]
                args[k] = t + sign * 1e-2 * d
                ends.append(f(*args))
        got, want = (grads[k].double() * d).sum(), (ends[0] - ends[1]) / 2e-2
        # step^2 / 6 of the third derivative, and 330 fp32 values of about 1 over the step
        assert abs(got - want) <= 2e-3 * (grads[k].double() * d).abs().sum()


def test_empty_and_changed_since():
    from paper_2607_26005_amd import memory
    x, w = torch.zeros(0, 16, device="cuda", requires_grad=True), torch.ones(16, device="cuda", requires_grad=True)
    y = memory.rms_norm(x, w)
    dx, dw = torch.autograd.grad(y.sum(), (x, w))
    assert y.shape == (0, 16) and dx.shape == (0, 16) and (dw == 0).all()
    assert memory.rms_norm_8bit(x.detach(), w.detach()).values().shape == (0, 16)
    x = torch.randn(3, 16, device="cuda", requires_grad=True)
    y, s = memory.rms_norm(x * 1, w, x * 2)
    with torch.no_grad():
        s.add_(1)
    with pytest.raises(RuntimeError, match="modified by an inplace"):
        y.sum().backward()


def test_in_place_and_beyond_the_rows():
    from paper_2607_26005_amd import memory, pictura
    for c, dtype in ((331, torch.bfloat16), (512, torch.float32), (16500, torch.float16)):
        x, r, w = _rows(1, 9, c, dtype), _rows(2, 9, c, dtype), _rand(3, c).cuda()
        y, s = memory.rms_norm(x, w, r)
        # sum over the residual, out over x
        r2, x2 = r.clone(), x.clone()
        pictura.pictura_rms_norm(x2, w, x2, r2, r2)
        assert torch.equal(x2, y) and torch.equal(r2, s)
        held = torch.full((11, c + 5), 7.0, dtype=dtype, device="cuda")
        pictura.pictura_rms_norm(x, w, held[1:10, 2:2 + c], None, r)
        assert torch.equal(held[1:10, 2:2 + c], y)
        held[1:10, 2:2 + c] = 7.0
        assert (held == 7.0).all()
        codes = torch.full((11, c + 5), 77, dtype=torch.int8, device="cuda")
        scales = torch.full((11,), 7.0, device="cuda")
        pictura.pictura_rms_norm_codes(x, w, codes[1:10, 2:2 + c], scales[1:10], None, r)
        assert torch.equal(codes[1:10, 2:2 + c], memory.rms_norm_8bit(x, w, r, dtype=torch.int8).codes)
        codes[1:10, 2:2 + c] = 77
        assert (codes == 77).all() and scales[0] == 7 and scales[10] == 7
        # the gradient over the one that arrived
        _, f = None, torch.empty(9, device="cuda")
        out = torch.empty_like(x)
        pictura.pictura_rms_norm(x, w, out, factors=f)
        dy, dw = _rows(5, 9, c, dtype), torch.empty_like(w)
        dx = torch.empty_like(x)
        pictura.pictura_rms_norm_gradient(x, w, f, dy, dx, dw)
        pictura.pictura_rms_norm_gradient(x, w, f, dy, dy, dw)
        assert torch.equal(dx, dy)


def test_streams_and_graphs():
    from paper_2607_26005_amd import memory, pictura
    x, r, w = _rows(1, 500, 520, torch.bfloat16), _rows(2, 500, 520, torch.bfloat16), _rand(3, 520).cuda()
    want = memory.rms_norm(x, w, r)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = memory.rms_norm(x, w, r)
    torch.cuda.current_stream().wait_stream(side)
    assert all(map(torch.equal, got, want))
    f, dx, dw, dy = torch.empty(500, device="cuda"), torch.empty_like(x), torch.empty_like(w), _rows(4, 500, 520, torch.bfloat16)
    y, s = torch.empty_like(x), torch.empty_like(x)

    def both():
        pictura.pictura_rms_norm(x, w, y, s, r, 1e-6, f)
        pictura.pictura_rms_norm_gradient(s, w, f, dy, dx, dw)
        return memory.rms_norm_8bit(x, w, r)

    both()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = both()
    for k in range(3):
        x.copy_(_rand(40 + k, 500, 520))
        now = both()
        want = [t.clone() for t in (y, s, f, dx, dw)]
        for t in (y, s, f, dx, dw):
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(map(torch.equal, (y, s, f, dx, dw), want))
        assert torch.equal(held.codes.view(torch.uint8), now.codes.view(torch.uint8)) and torch.equal(held.scales, now.scales)


def test_offsets_beyond_32_bits():
    from paper_2607_26005_amd import memory
    far = 1 << 32
    base = torch.empty(far + 4096, dtype=torch.float16, device="cuda")
    x, w = _rows(1, 2, 96, torch.float16), torch.ones(96, device="cuda")
    view = torch.as_strided(base, (2, 96), (far, 1))
    view.copy_(x)
    assert torch.equal(memory.rms_norm(view, w), memory.rms_norm(x, w))


@pytest.mark.parametrize("kind", [torch.float8_e4m3fn, torch.int8])
def test_codes_lose_no_gradient_without_a_word(kind):
    """The sum of a norm to 8 bits hands on its gradient; its codes, which have none, raise
    where one would arrive."""
    from paper_2607_26005_amd import memory
    x, w, r = (_rand(k, *s).cuda() for k, s in ((1, (6, 40)), (2, (40,)), (3, (6, 40))))
    want = memory.rms_norm_8bit(x, w, r, dtype=kind)
    assert not any(t.requires_grad for t in want) and not want.values().requires_grad
    wants = [t.clone().requires_grad_() for t in (x, w, r)]
    x1, w1, r1 = wants
    dy = _rand(4, 6, 40).cuda()
    held = memory.rms_norm_8bit(x1, w1, r1, dtype=kind)
    assert torch.equal(held.codes.detach().view(torch.uint8), want.codes.view(torch.uint8))
    assert torch.equal(held.scales, want.scales) and torch.equal(held.sum, want.sum)
    dx, dr = torch.autograd.grad(held.sum, (x1, r1), dy)
    assert torch.equal(dx, dy) and torch.equal(dr, dy)
    both, = torch.autograd.grad(memory.rms_norm_8bit(x1, w, x1, dtype=kind).sum, x1, dy)   # the same tensor twice
    assert torch.equal(both, 2 * dy)
    twice = torch.autograd.grad(memory.rms_norm_8bit(x1 * 1, w, r, dtype=kind).sum.pow(3).sum(), x1, create_graph=True)[0]
    again, = torch.autograd.grad(twice.sum(), x1)
    assert torch.allclose(again, 6 * (x + r), rtol=1e-5, atol=1e-6)
    for a in ((x1, w, r), (x, w1, r), (x, w, r1), (x1, w1, None)):
        held = memory.rms_norm_8bit(*a, dtype=kind)
        assert a[2] is None or held.sum.requires_grad == (a[1] is w)
        with pytest.raises(RuntimeError, match="codes and scales have no gradient"):
            held.scales.sum().backward()
        with pytest.raises(RuntimeError, match="have no gradient"):
            held.values().sum().backward()
        if kind is torch.float8_e4m3fn:
            with pytest.raises(RuntimeError, match="codes and scales have no gradient"):
                held.codes.float().sum().backward()
        free = memory.RowCodes(held.codes.detach(), held.scales.detach(), None).values()
        assert torch.equal(free, held.values()) and not free.requires_grad
    assert all(t.grad is None for t in wants)
    with torch.no_grad():
        assert not any(t is not None and t.requires_grad for t in memory.rms_norm_8bit(x1, w1, r1, dtype=kind))
