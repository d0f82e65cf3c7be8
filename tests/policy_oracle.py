"""The policy's operators in 64 bits, plainly, on the host."""
import numpy as np


def kept_weights(logits, mask=None, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """(probabilities drawn from, how near a filter's decision was to going the
    other way) of one row, in float64; None where there is nothing to draw."""
    x = np.asarray(logits, np.float64).copy()
    allowed = np.ones(len(x), bool) if mask is None else np.asarray(mask, bool)
    x[~allowed] = -np.inf
    if np.isnan(x).any() or (x == np.inf).any() or not (x > -np.inf).any() or not temperature >= 0:
        return None, np.inf
    order = np.argsort(-x, kind="stable")
    if temperature == 0:
        p = np.zeros(len(x))
        p[order[0]] = 1.0
        return p, np.inf
    with np.errstate(over="ignore"):
        w = np.exp((x - x.max()) / temperature)
    ws, near = w[order].copy(), np.inf
    if 0 < top_k < len(x):
        ws[top_k:] = 0.0
    if top_p < 1:
        c = np.cumsum(ws) / ws.sum()
        n = 1 + int(np.searchsorted(c, max(top_p, 0.0), side="left"))
        near = np.abs(c - top_p).min()
        ws[n:] = 0.0
    if min_p > 0:
        near = min(near, np.abs(ws - min_p).min())
        ws[ws < min(min_p, 1.0)] = 0.0
    p = np.zeros(len(x))
    p[order] = ws / ws.sum()
    return p, near


def draw(p, u):
    """(action, distance of u from the nearest edge of the action's interval)."""
    c = np.cumsum(p)
    a = int(np.searchsorted(c, u * c[-1], side="right"))
    edges = np.concatenate([[0.0], c])
    return a, float(np.abs(edges[(edges > 0) & (edges < c[-1])] - u).min()) if np.count_nonzero(p) > 1 else 1.0


def policy_loss(logits, values, actions, old_logp, advantages, returns, old_values=None, weights=None, mask=None,
                temperature=1.0, clip=0.2, value_clip=0.0, value_coef=0.5, entropy_coef=0.01, normalize=False,
                denominator=0.0, value_only=False):
    """Stats, d logits, d values in float64 (value_only: the loss alone)."""
    f = lambda a: np.asarray(a, np.float64)
    z, v = f(logits).copy(), f(values)
    N, A = z.shape
    act = np.asarray(actions)
    w = np.ones(N) if weights is None else f(weights).copy()
    w[(act < 0) | (act >= A)] = 0.0
    used = w != 0
    if mask is not None:
        z[~np.broadcast_to(np.asarray(mask, bool), z.shape)] = -np.inf
    stats, dz, dv = np.zeros(6), np.zeros((N, A)), np.zeros(N)
    den = denominator if denominator else w[used].sum()
    if not used.any():
        return 0.0 if value_only else (stats, dz, dv)
    adv = f(advantages).copy()
    if normalize:
        mean = (w[used] * adv[used]).sum() / w[used].sum()
        std = np.sqrt((w[used] * (adv[used] - mean) ** 2).sum() / w[used].sum())
        adv = (adv - mean) / (std + 1e-8)
    terms = np.zeros((N, 5))
    for n in np.flatnonzero(used):
        top = z[n].max()
        d = (z[n] - top) / temperature if top > -np.inf else np.full(A, -np.inf)
        e = np.exp(d)
        S = e.sum()
        p = e / S if S > 0 else e
        lp = np.where(e > 0, d - (np.log(S) if S > 0 else 0.0), 0.0)
        H = -(p * lp).sum()
        logp = lp[act[n]] if e[act[n]] > 0 else -np.inf
        diff = logp - f(old_logp)[n]
        r = np.exp(diff)
        un, cl = r * adv[n], np.clip(r, 1 - clip, 1 + clip) * adv[n]
        g = -un if un <= cl else 0.0
        err = dvn = v[n] - f(returns)[n]
        if value_clip > 0:
            move = v[n] - f(old_values)[n]
            far = f(old_values)[n] + np.clip(move, -value_clip, value_clip) - f(returns)[n]
            if abs(move) > value_clip and abs(far) > abs(err):
                err, dvn = far, 0.0
        terms[n] = -min(un, cl), err * err / 2, H, r - 1 - diff, not 1 - clip <= r <= 1 + clip
        dz[n] = entropy_coef * p * (lp + H) - g * p
        dz[n, act[n]] += g
        dz[n] *= w[n] / den / temperature
        dv[n] = value_coef * dvn * w[n] / den
    stats[1:] = (w[used, None] * terms[used]).sum(0) / den
    stats[0] = stats[1] + value_coef * stats[2] - entropy_coef * stats[3]
    return stats[0] if value_only else (stats, dz, dv)


def adamw(param, grad, m, v, step, lr, betas, eps, weight_decay, factor=1.0):
    """(param, m, v) after a step, in float64."""
    p, g, m, v = (np.asarray(a, np.float64) for a in (param, grad, m, v))
    g = g * factor
    m = betas[0] * m + (1 - betas[0]) * g
    v = betas[1] * v + (1 - betas[1]) * g * g
    p = p * (1 - lr * weight_decay)
    return p - lr * (m / (1 - betas[0] ** step)) / (np.sqrt(v / (1 - betas[1] ** step)) + eps), m, v


def _blocks(x):
    n = len(x)
    b = np.zeros((-(-n // 256), 256))
    b.reshape(-1)[:n] = x
    return b


def moment_values(codes, scales, second):
    c = _blocks(np.asarray(codes, np.float64))
    x = (c / 255) ** 4 if second else c * np.abs(c) / 127.0 ** 2
    return (x * np.asarray(scales, np.float64)[:, None]).reshape(-1)[:len(codes)]


def moment_positions(x, second):
    """Where each value lies on its code's scale, before rounding, and the scales."""
    b = _blocks(np.asarray(x, np.float64))
    s = np.abs(b).max(1)
    s[s < 2.0 ** -90] = 0.0
    r = np.divide(np.abs(b), s[:, None], out=np.zeros_like(b), where=s[:, None] > 0)
    q = 255 * r ** 0.25 if second else 127 * np.sqrt(r) * np.sign(b)
    return q.reshape(-1)[:len(x)], s
