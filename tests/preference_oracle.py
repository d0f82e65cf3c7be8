"""The preference loss on the host in 64 bits, its gradient by autograd from the loss, and
bounds of what fp32 arithmetic may leave (u = 2^-24).

A row's log-probability is (x - top) - log S - ref in fp32: u of each difference and of the
logarithm (which is off by 2 u), and the relative error of S, whose terms are off by 4 u and
u |d| each and whose sum takes `depth` additions one after the other.  Sequences add those up
in fp64; a factor c then moves by the margin's error times the slope of the sigmoid."""
import math

import torch

U = 2.0 ** -24


def preference(logits, actions, offsets, ref=None, weights=None, mask=None, beta=0.1, smoothing=0.0, average=False,
               denominator=0.0):
    """{name: (value, bound)} of stats, ratios, dlogits."""
    z = logits.detach().cpu().double().requires_grad_()
    N, A = z.shape
    a = actions.cpu()
    off = offsets.cpu().clamp(0, N).tolist()
    P = len(off) // 2
    allowed = torch.ones(N, A, dtype=torch.bool) if mask is None else mask.cpu().bool().expand(N, A)
    allowed = allowed & (z.detach() != -math.inf)
    counts = (a >= 0) & (a < A) & allowed.any(1)
    taken = a.clamp(0, A - 1)[:, None]
    safe = torch.where(allowed, z, torch.full_like(z, -1e300))
    safe = torch.where(counts[:, None], safe, torch.zeros_like(safe))
    logp = safe.log_softmax(1).gather(1, taken)[:, 0]
    out_of = counts & ~allowed.gather(1, taken)[:, 0]
    r = torch.zeros(N, dtype=torch.float64) if ref is None else ref.cpu().double()
    row = torch.where(counts, logp - r, torch.zeros_like(logp))
    w = torch.ones(P, dtype=torch.float64) if weights is None else weights.cpu().double()
    omega = denominator or w.sum().item()
    # errors of the rows
    with torch.no_grad():
        x = torch.where(allowed, z, torch.full_like(z, -math.inf))
        top = x.max(1, keepdim=True).values.clamp(min=-1e300)
        d = (x - top).abs()
        p = torch.where(allowed, safe.softmax(1), torch.zeros_like(safe))
        depth = max(16, A // 64) + 12
        far = torch.where(allowed & (p > 0), d, torch.zeros_like(d))
        eS = U * (4 + depth + (p * far).sum(1))
        logs = (x - top).exp().sum(1).log()
        logs = torch.where(counts, logs, torch.zeros_like(logs))
        da = far.gather(1, taken)[:, 0]
        e_row = torch.where(counts & ~out_of, eS + U * (2 * da + 4 * logs.abs() + row.abs() + r.abs() + logp.abs()), torch.zeros_like(row))
    D, eD, scale = [], [], []
    for s in range(2 * P):
        lo, hi = off[s], max(off[s], off[s + 1])
        n = int(counts[lo:hi].sum())
        part = 1 / n if average and n > 1 else 1.0
        some = row[lo:hi].sum() * part
        D.append(torch.where(out_of[lo:hi].any(), torch.full_like(some, -math.inf), some))
        eD.append(e_row[lo:hi].sum() * part)
        scale.append(part)
    zero = torch.zeros((), dtype=torch.float64)
    loss = stats = zero
    bound_stats, terms = [0.0] * 4, [0.0] * 4
    c, ec = torch.zeros(N, dtype=torch.float64), torch.zeros(N, dtype=torch.float64)
    up_to = lambda t: t.clamp(min=0) + torch.log1p((-t.abs()).exp())
    for k in range(P):
        if w[k] == 0 or omega == 0:
            continue
        m = beta * (D[2 * k] - D[2 * k + 1])
        em = (beta * (eD[2 * k] + eD[2 * k + 1])).item() + 2 * U * m.abs().item()
        one = (1 - smoothing) * up_to(-m) + (smoothing * up_to(m) if smoothing else 0.0)
        wk = w[k].item() / omega
        mm = m.item()
        for j, v in enumerate((one.item(), beta * D[2 * k].item(), beta * D[2 * k + 1].item(), float(mm > 0))):
            terms[j] += wk * v
        for j, e in enumerate((em, beta * eD[2 * k].item(), beta * eD[2 * k + 1].item(), 0.0)):
            bound_stats[j] += abs(wk) * e
        sig = 1 / (1 + math.exp(-mm)) if mm > -700 else 0.0
        g = wk * beta * (smoothing * sig - (1 - smoothing) * (1 - sig))
        eg = abs(wk) * beta * min(1.0, 1.1 * sig * (1 - sig) + em) * em + 3 * U * abs(g)
        for s, sign in ((2 * k, 1.0), (2 * k + 1, -1.0)):
            lo, hi = off[s], max(off[s], off[s + 1])
            c[lo:hi], ec[lo:hi] = sign * g * scale[s], eg * scale[s]
    delta = torch.zeros(N, A, dtype=torch.float64).scatter_(1, taken, 1.0)
    delta = torch.where(allowed, delta, torch.zeros_like(delta))
    live = (counts & (c != 0))[:, None]
    dl = torch.where(live, c[:, None] * (delta - p), torch.zeros_like(p))
    bl = torch.where(live, ec[:, None] * (delta + p) + c.abs()[:, None] * (3 * U * delta + p * (eS[:, None] + U * (8 + far))),
                     torch.zeros_like(p)).nan_to_num(0.0)
    D, eD = torch.stack(D) if P else torch.zeros(0), torch.stack(eD) if P else torch.zeros(0)
    return {"stats": (torch.tensor(terms, dtype=torch.float64), torch.tensor(bound_stats, dtype=torch.float64)),
            "ratios": (D.detach().double(), eD.double()), "dlogits": (dl.detach(), bl.detach())}


def by_autograd(logits, actions, offsets, ref, beta):
    """The gradient from the loss alone (all rows count, sums, no weights)."""
    z = logits.detach().cpu().double().requires_grad_()
    row = z.log_softmax(1).gather(1, actions.cpu()[:, None])[:, 0] - ref.cpu().double()
    o = offsets.tolist()
    D = torch.stack([row[i:j].sum() for i, j in zip(o, o[1:])])
    loss = -torch.nn.functional.logsigmoid(beta * (D[0::2] - D[1::2])).mean()
    return loss.detach(), torch.autograd.grad(loss, z)[0]
