"""Plain 64-bit forms of the memory's operators on the host, step by step, with bounds of
the error that fp32 arithmetic may leave.

The bounds are running ones, u = 2^-24: a rounded operation adds u of its result, the
gate's two parts come to within 10 u of their own (a hardware exponential off by up to a
unit, 2 u; two roundings of its correction; 1 + e, the reciprocal off by a unit, their
product and the difference from 1, with the exponential's error passed on), and errors
travel through the recurrence with the factors of the values.  Magnitudes stand for
values, so that the bounds hold for any split of the steps.

Gates of 16 bits: the product |g| log2 e is rounded once, by u of itself, and the constant
by 0.23 u, which in exp(-|g|) is a relative 1.23 |g| u, and no more than that in either part
(the larger one, 1 - m, has it times m / (1 - m) <= 1)."""
import torch

U = 2.0 ** -24
GATE = 10


def _gate(g, dtype):
    """Units that a gate's parts may be off by."""
    return GATE if dtype == torch.float32 else GATE + 1.23 * g.abs()


def half_step(t, dtype):
    """Half a unit of `dtype` at values t: what one rounding may change (subnormals too)."""
    info = torch.finfo(dtype)
    return t.abs() * (info.eps / 2) + info.smallest_normal * info.eps / 2


def scan(gates, inputs, state=None, resets=None):
    """(h, last, bound of h, bound of last) of [batch, steps, channels] tensors."""
    g, x = gates.detach().cpu().double(), inputs.detach().cpu().double()
    B, T, C = x.shape
    h = torch.zeros(B, C, dtype=torch.float64) if state is None else state.detach().cpu().double()
    A, e = h.abs(), torch.zeros_like(h)
    out, bound, mags = torch.empty_like(x), torch.empty_like(x), torch.empty_like(x)
    for t in range(T):
        a, b = g[:, t].sigmoid(), (-g[:, t]).sigmoid()
        if resets is not None:
            began = resets.cpu().bool()[:, t, None]
            h, A, e = (torch.where(began, torch.zeros_like(v), v) for v in (h, A, e))
        off = _gate(g[:, t], gates.dtype)
        e = a * e + U * ((off + 4) * a * A + (off + 4) * b * x[:, t].abs())
        h, A = a * h + b * x[:, t], a * A + b * x[:, t].abs()
        e = e + U * A
        out[:, t], bound[:, t], mags[:, t] = h, e, A
    return out, h, bound, e


def scan_gradient(gates, inputs, state, resets, dout, dlast):
    """(dgates, dinputs, dstate) and the bounds of the three."""
    g, x, dy = (t.detach().cpu().double() for t in (gates, inputs, dout))
    B, T, C = x.shape
    h, last, eh, _ = scan(gates, inputs, state, resets)
    mag = scan(gates, inputs.abs(), None if state is None else state.abs(), resets)[0]
    first = torch.zeros(B, C, dtype=torch.float64) if state is None else state.detach().cpu().double()
    c = torch.zeros(B, C, dtype=torch.float64) if dlast is None else dlast.detach().cpu().double()
    cm, ec = c.abs(), torch.zeros_like(c)
    dg, dx, bg, bx = (torch.empty_like(x) for _ in range(4))
    zero = torch.zeros_like(c)
    for t in range(T - 1, -1, -1):
        a, b = g[:, t].sigmoid(), (-g[:, t]).sigmoid()
        G, Gm = dy[:, t] + c, dy[:, t].abs() + cm
        eG = ec + U * Gm
        before, bm, eb = (h[:, t - 1], mag[:, t - 1], eh[:, t - 1]) if t else (first, first.abs(), zero)
        if resets is not None:
            began = resets.cpu().bool()[:, t, None]
            before, bm, eb = (torch.where(began, zero, v) for v in (before, bm, eb))
        d, dm = before - x[:, t], bm + x[:, t].abs()
        off = _gate(g[:, t], gates.dtype)
        dx[:, t], bx[:, t] = b * G, b * eG + (off + 2) * U * b * Gm
        dg[:, t] = a * b * G * d
        bg[:, t] = a * b * (dm * eG + Gm * (eb + U * dm) + (2 * off + 4) * U * Gm * dm)
        c, cm, ec = a * G, a * Gm, a * eG + (off + 4) * U * a * Gm
        if resets is not None:
            c, cm, ec = (torch.where(began, zero, v) for v in (c, cm, ec))
    return (dg, dx, c), (bg, bx, ec)


# --- the norm ---------------------------------------------------------------------

def norm(x, weight, residual=None, eps=1e-6):
    """(what is normed in x's type, y, factor q [rows, 1]) of [rows, width] tensors."""
    s = x.detach().cpu()
    if residual is not None:
        s = (s.float() + residual.detach().cpu().float()).to(s.dtype)
    q = 1 / (s.double().pow(2).mean(1, keepdim=True) + eps).sqrt()
    return s, s.double() * q * weight.detach().cpu().double(), q


def norm_codes(x, weight, residual, eps, dtype):
    """(codes, scales) by the operator's own fp32 steps, of a mean in 64 bits."""
    s, _, q = norm(x, weight, residual, eps)
    y = (s.float() * q.float()) * weight.cpu().float()
    most = 127.0 if dtype == torch.int8 else 448.0
    top = y.abs().amax(1)
    none = top < 2.0 ** -100
    up = torch.where(none, torch.zeros_like(top), top.reciprocal() * most)
    code = y * up[:, None]
    code = code.round().to(torch.int8) if dtype == torch.int8 else code.to(dtype)
    return code, torch.where(none, torch.zeros_like(top), top / most)


def norm_gradient(s, weight, eps, dout, dsum):
    """(dx, dweight) and their bounds.  The kernels' sums are of 70 terms one after the other
    at most, and of 10 levels of lanes and waves; those over rows of all rows at most."""
    s, w, dy = (t.detach().cpu().double() for t in (s, weight, dout))
    q = 1 / (s.pow(2).mean(1, keepdim=True) + eps).sqrt()
    u, k = s * q, dy * w
    c, cm = (k * u).mean(1, keepdim=True), (k * u).abs().mean(1, keepdim=True)
    dx = q * (k - u * c)
    size = q * (k.abs() + u.abs() * c.abs())
    bound = 8 * U * size + q * u.abs() * 90 * U * cm
    if dsum is not None:
        dx = dx + dsum.detach().cpu().double()
    bound = bound + U * dx.abs()
    return (dx, (dy * u).sum(0)), (bound, (s.shape[0] + 6) * U * (dy * u).abs().sum(0))
