"""The policy's operators as cases that can be timed and compared.

What follows the image encoder in a training process: actions drawn from the
policy head's logits (temperature, top-k, top-p, min-p, from given random
numbers), the clipped policy loss with its gradient, and the AdamW step over
all weight tensors with its moments in 32 or in 8 bits.  `run` computes them in
plain torch operations, or with `own` through the framework's entry points.

A case: `op` is "sample", "loss" or "adamw".  sample and loss: `rows`
(decisions), `actions` (the head's width), `dtype` of the logits, `pad` (further
columns of the head's matrix behind the logits: the rows are that much further
apart), `mask` (a truth value per action).  sample: `per_row` (each row has its
own temperature and filters, spread around the case's) and the filters
themselves (0 or 1: off).  loss: `options` (value clipping, row weights and
normalised advantages).  adamw: `tensors` (0: the policy's own weights) of
`total` elements together, `dtype` of the weights, `grad_dtype`, `bits`,
`max_norm` (0: no clipping of the gradient).
"""
import math
import random

import torch

own = False

_DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
_BLOCK = 256        # elements of one scale of an 8-bit moment
_ONE = 1 << 31      # weight of a row's largest logit


def _sample(name, rows, actions, dtype="f32", pad=0, mask=False, per_row=False, temperature=1.0, top_k=0, top_p=1.0,
            min_p=0.0):
    return dict(name=name, op="sample", rows=rows, actions=actions, dtype=dtype, pad=pad, mask=mask, per_row=per_row,
                temperature=temperature, top_k=top_k, top_p=top_p, min_p=min_p)


def _loss(name, rows, actions, dtype="f32", pad=0, mask=False, options=False):
    return dict(name=name, op="loss", rows=rows, actions=actions, dtype=dtype, pad=pad, mask=mask, options=options)


def _adamw(name, tensors, total, dtype="f32", grad_dtype="f32", bits=32, max_norm=0.0):
    return dict(name=name, op="adamw", tensors=tensors, total=total, dtype=dtype, grad_dtype=grad_dtype, bits=bits,
                max_norm=max_norm)


def listed():
    return [
        # the tiny world's eight agents choose among 4 x 3 motions: the call's latency
        _sample("act_tiny", 8, 12),
        # the headline step's 1,024 x 64 agents, some motions not allowed, logits beside the value in the head's output
        _sample("act_training_step", 65536, 12, pad=1, mask=True),
        # one ego asks for one of many trajectory tokens: latency again, over a long row
        _sample("plan_one_ego", 1, 16385, top_k=50, top_p=0.95, temperature=0.8),
        # one chunk of egos with their own settings
        _sample("plan_chunk", 2048, 4099, "bf16", per_row=True, top_k=64, top_p=0.95, min_p=0.02, temperature=0.8),
        # a large token vocabulary with the nucleus alone
        _sample("plan_large_vocabulary", 512, 65536, top_p=0.9),
        # one chunk of 2,048 egos in gradient accumulation
        _loss("loss_chunk", 2048, 12),
        # the whole minibatch: filtered rows, clipped values, normalised advantages
        _loss("loss_minibatch", 65536, 12, pad=1, mask=True, options=True),
        # trajectory tokens in bfloat16, rows of an odd length
        _loss("loss_tokens", 2047, 16381, "bf16", options=True),
        # the encoder and the actor-critic on it, with the gradient's norm clipped
        _adamw("step_policy", 0, 0, max_norm=0.5),
        # the same with the moments in 8 bits
        _adamw("step_policy_8bit", 0, 0, bits=8),
        # a larger network of many tensors, gradients in bfloat16
        _adamw("step_many_tensors", 300, 50_000_000, grad_dtype="bf16", max_norm=1.0),
        # a large network in bfloat16, moments in 8 bits
        _adamw("step_large_8bit", 64, 128_000_000, dtype="bf16", grad_dtype="bf16", bits=8),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["sample", "sample", "loss", "adamw"])
    dtype = rng.choice(["f32", "f32", "bf16", "f16"])
    if op == "adamw":
        total = _log(rng, 20_000, 100_000_000)
        tensors = min(_log(rng, 2, 400), total // 64)
        bits = rng.choice([32, 8])
        # (8-bit codes repeat to the bit only where the gradient's scale does: a clipped gradient's last bit goes by the
        # order of the norm's sum)
        c = _adamw("", tensors, total, rng.choice(["f32", "bf16"]), rng.choice(["f32", "bf16", "f16"]), bits,
                   0.0 if bits == 8 else rng.choice([0.0, 0.5, 1.0]))
    else:
        actions = rng.choice([2, 7, 12, 27, 64]) if rng.random() < 0.3 else _log(rng, 3, 65536)
        rows = _log(rng, 1, min(65536, (1 << 25) // actions))
        pad, mask = rng.choice([0, 0, 1, 5]), rng.random() < 0.3
        if op == "loss":
            c = _loss("", rows, actions, dtype, pad, mask, rng.random() < 0.5)
        else:
            c = _sample("", rows, actions, dtype, pad, mask, rng.random() < 0.3,
                        rng.choice([1.0, 1.0, round(rng.uniform(0.3, 2.0), 2)]),
                        rng.choice([0, 0, _log(rng, 1, 512)]), rng.choice([1.0, 1.0, round(rng.uniform(0.3, 0.99), 3)]),
                        rng.choice([0.0, 0.0, round(rng.uniform(0.001, 0.2), 4)]))
    del c["name"]
    return c


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------

class _State:
    pass


def _head(case, g):
    """The head's output matrix: the logits, then `pad` further columns."""
    N, A = case["rows"], case["actions"]
    # a dozen motions: a policy some way into training; many tokens: a long tail under a few likely ones
    spread = 1.5 if A <= 64 else 2.5
    return (torch.randn(N, A + case["pad"], generator=g, device="cuda") * spread).to(_DTYPES[case["dtype"]])


def _mask(case, g):
    if not case["mask"]:
        return None
    m = torch.rand(case["rows"], case["actions"], generator=g, device="cuda") < 0.8
    m[:, 0] = True   # keeping the lane and the speed is always allowed
    return m


def _prepare_sample(s, case, g):
    N = case["rows"]
    s.logits = _head(case, g)[:, :case["actions"]]
    s.mask = _mask(case, g)
    s.uniform = torch.rand(N, generator=g, device="cuda")
    s.settings = {k: case[k] for k in ("temperature", "top_k", "top_p", "min_p")}
    if case["per_row"]:
        f = torch.rand(4, N, generator=g, device="cuda") + 0.5
        s.settings["temperature"] = case["temperature"] * f[0]
        s.settings["top_k"] = (case["top_k"] * f[1]).ceil().to(torch.int32)
        if case["top_p"] < 1:
            s.settings["top_p"] = 1 - (1 - case["top_p"]) * f[2].clamp(max=1)
        s.settings["min_p"] = case["min_p"] * f[3]


def _prepare_loss(s, case, g):
    N, A = case["rows"], case["actions"]
    head = _head(case, g)
    s.logits = head[:, :A]
    s.values = head[:, A].float() if case["pad"] and case["dtype"] != "f32" else \
        head[:, A] if case["pad"] else torch.randn(N, generator=g, device="cuda")
    s.mask = _mask(case, g)
    z = s.logits.float() if s.mask is None else s.logits.float().masked_fill(~s.mask, -math.inf)
    s.actions = (z - (-torch.rand(N, A, generator=g, device="cuda").clamp_min(1e-20).log()).log()).argmax(1)
    z = z.double()
    logp = (z - z.logsumexp(1, keepdim=True)).gather(1, s.actions[:, None])[:, 0]
    # how far the policy moved since the rollout; kept off the clip's edges, where a last bit decides
    moved = torch.randn(N, generator=g, device="cuda", dtype=torch.float64) * 0.15
    r = moved.exp()
    moved = torch.where(((r - 0.8).abs() < 1e-4) | ((r - 1.2).abs() < 1e-4), 0.05, moved)
    s.old_logp = (logp - moved).float()
    s.advantages = torch.randn(N, generator=g, device="cuda") * 0.7 + 0.1
    s.returns = s.values + torch.randn(N, generator=g, device="cuda") * 0.5
    s.old_values = s.weights = None
    s.value_clip, s.normalize = 0.0, False
    if case["options"]:
        s.old_values = s.values + torch.randn(N, generator=g, device="cuda") * 0.2
        s.weights = (torch.rand(N, generator=g, device="cuda") < 0.75).float()   # the advantage filter
        s.weights[0] = 1.0
        s.value_clip, s.normalize = 0.2, True


def _sizes(case):
    if case["tensors"] == 0:
        # the encoder at the paper's four cameras (convolutions, queries, attention, projection), then a hidden width
        # of 512 four times and the two heads
        chans, w = (12, 32, 64, 64, 128, 128), 128
        out = [n for i in range(5) for n in (9 * chans[i] * chans[i + 1], chans[i + 1])]
        out += [4 * 16 * w, 3 * w * w, 3 * w, w * w, w, w * w, w]
        return out + [512 * 512, 512] * 4 + [12 * 512, 12, 512, 1]
    rng = random.Random(case["tensors"] * 1_000_003 + case["total"])
    part = [math.exp(rng.uniform(0.0, 5.0)) for _ in range(case["tensors"])]
    return [max(1, int(case["total"] * x / sum(part))) for x in part]


def _stands(q, power, levels, scale):
    """What an 8-bit moment's levels stand for: (q / levels)^power of the block's scale."""
    q = q * q.abs() if power == 2 else (q * q) * (q * q)
    return (q.view(-1, _BLOCK) * (scale * (1.0 / levels ** power))[:, None]).view(-1)


def _levels(x, power, levels):
    """An 8-bit moment's levels (whole numbers) and the scale of each block."""
    x = x.view(-1, _BLOCK)
    scale = x.abs().amax(1)
    scale = torch.where(scale < 2.0 ** -90, torch.zeros_like(scale), scale)
    inv = torch.where(scale > 0, 1.0 / scale, torch.zeros_like(scale))
    y = (x.abs() * inv[:, None]).sqrt()
    if power == 4:
        y = y.sqrt()
    q = (y * float(levels)).round().clamp(max=float(levels))
    q = torch.where(x < 0, -q, q) if power == 2 else torch.where((x > 0) & (scale[:, None] > 0), q.clamp(min=1.0), q)
    return q.view(-1), scale


def _prepare_adamw(s, case, g):
    sizes = _sizes(case)
    # every tensor starts on a whole block of one storage
    starts, at = [], 0
    for n in sizes:
        starts.append(at)
        at += -(-n // _BLOCK) * _BLOCK
    inside = torch.zeros(at + 1, dtype=torch.int32, device="cuda")
    inside.index_add_(0, torch.tensor(starts, device="cuda"), torch.ones(len(sizes), dtype=torch.int32, device="cuda"))
    inside.index_add_(0, torch.tensor([b + n for b, n in zip(starts, sizes)], device="cuda"),
                      torch.full((len(sizes),), -1, dtype=torch.int32, device="cuda"))
    inside = inside.cumsum(0)[:at] > 0
    rand = lambda scale: torch.where(inside, torch.randn(at, generator=g, device="cuda") * scale, 0.0)
    s.param = rand(0.05).to(_DTYPES[case["dtype"]])
    s.grad = rand(1e-3).to(_DTYPES[case["grad_dtype"]])
    s.m, s.v = rand(3e-4), rand(1e-3).square()
    s.bits, s.max_norm, s.step = case["bits"], case["max_norm"], 100
    if s.bits == 8:
        qm, s.m_scale = _levels(s.m, 2, 127)
        qv, s.v_scale = _levels(s.v, 4, 255)
        s.m_code, s.v_code = qm.to(torch.int8), qv.to(torch.uint8)
    s.lr, s.betas, s.eps, s.decay = 5e-4, (0.9, 0.999), 1e-8, 0.01
    s.opt = None
    if own:   # the optimizer object that a program keeps, its state where the plain form has it
        from paper_2607_26005_amd import policy
        cut = lambda t: [t[b:b + n] for b, n in zip(starts, sizes)]
        part = lambda t: [t[b // _BLOCK:b // _BLOCK + -(-n // _BLOCK)] for b, n in zip(starts, sizes)]
        params = [torch.nn.Parameter(p) for p in cut(s.param)]
        s.grads = cut(s.grad)
        s.opt = policy.AdamW(params, lr=s.lr, betas=s.betas, eps=s.eps, weight_decay=s.decay, bits=s.bits,
                             max_norm=s.max_norm or None)
        names = ("exp_avg", "exp_avg_sq") if s.bits == 32 else ("exp_avg", "exp_avg_sq", "exp_avg_scale",
                                                               "exp_avg_sq_scale")
        held = [cut(s.m), cut(s.v)] if s.bits == 32 else [cut(s.m_code), cut(s.v_code), part(s.m_scale), part(s.v_scale)]
        for p, *t in zip(params, *held):
            s.opt.state[p].update(zip(names, t), step=s.step)
        if s.bits == 8:
            s.moments = cut(s.m), cut(s.v)


def prepare(case, seed):
    s = _State()
    s.op = case["op"]
    g = torch.Generator("cuda").manual_seed(seed)
    {"sample": _prepare_sample, "loss": _prepare_loss, "adamw": _prepare_adamw}[s.op](s, case, g)
    return s


# ---------------------------------------------------------------------------
# plain forms
# ---------------------------------------------------------------------------

def _column(x, like, dtype):
    return (x if isinstance(x, torch.Tensor) else torch.full_like(like, x, dtype=torch.float32)).to(dtype)[:, None]


def _share(total, x):
    """floor(total * floor(x 2^31) / 2^31) of whole numbers, x in [0, 1)."""
    m = (x.clamp(0.0, 1.0 - 2.0 ** -24) * float(_ONE)).to(torch.int64)
    return (total >> 32) * m * 2 + ((total & 0xFFFFFFFF) * m >> 31)


def _plain_sample(logits, uniform, mask, temperature, top_k, top_p, min_p):
    x = logits.float()
    if mask is not None:
        x = x.masked_fill(~mask, -math.inf)
    top = x.amax(1, keepdim=True)
    e = ((x - top) / _column(temperature, uniform, torch.float32)).exp()
    w = (e * float(_ONE)).round().to(torch.int64)
    filtered = [isinstance(v, torch.Tensor) or v != off for v, off in ((top_k, 0), (top_p, 1.0), (min_p, 0.0))]
    if filtered[0] or filtered[1]:
        order = x.sort(dim=1, descending=True, stable=True).indices   # equal logits: the lowest index first
        ws = w.gather(1, order)
        if filtered[0]:
            k = _column(top_k, uniform, torch.int64)
            ws = ws * ((torch.arange(ws.shape[1], device=ws.device) < k) | (k <= 0))
        if filtered[1]:
            p = _column(top_p, uniform, torch.float32)
            need = _share(ws.sum(1, keepdim=True), p).clamp_min(1)
            ws = ws * ((ws.cumsum(1) - ws < need) | (p >= 1))
        w = torch.zeros_like(w).scatter_(1, order, ws)
    if filtered[2]:
        least = (_column(min_p, uniform, torch.float32) * float(_ONE)).ceil().to(torch.int64)
        w = w * (w >= least)
    c = w.cumsum(1)
    total = c[:, -1:]
    action = (c <= _share(total, uniform[:, None])).sum(1, keepdim=True)
    logp = (w.gather(1, action).float() / total.float()).log()
    return action[:, 0], logp[:, 0]


def _plain_loss(s):
    x = s.logits.float()
    if s.mask is not None:
        x = x.masked_fill(~s.mask, -math.inf)
    N = x.shape[0]
    w = torch.ones_like(s.returns) if s.weights is None else s.weights
    total = w.sum()
    adv = s.advantages
    if s.normalize:
        mean = (w * adv).sum() / total
        adv = (adv - mean) / ((w * (adv - mean).square()).sum() / total).sqrt().add(1e-8)
    d = x - x.amax(1, keepdim=True)
    e = d.exp()
    S = e.sum(1, keepdim=True)
    p, log_s = e / S, S.log()
    lp = torch.where(e > 0, d - log_s, torch.zeros_like(d))
    H = -(p * lp).sum(1)
    at = s.actions[:, None]
    diff = (d.gather(1, at) - log_s)[:, 0] - s.old_logp
    r = diff.exp()
    un, cl = r * adv, r.clamp(1 - 0.2, 1 + 0.2) * adv
    pg = -torch.minimum(un, cl)
    g = torch.where(un <= cl, -un, torch.zeros_like(un))
    v, R = s.values, s.returns
    dv = v - R
    err = dv
    if s.value_clip > 0:
        move = v - s.old_values
        far = s.old_values + move.clamp(-s.value_clip, s.value_clip) - R
        use = (move.abs() > s.value_clip) & (far.abs() > dv.abs())
        err = torch.where(use, far, dv)
        dv = torch.where(use, torch.zeros_like(dv), dv)
    vl = 0.5 * err.square()
    mean = lambda t: (w * t).sum() / total
    parts = [mean(pg), mean(vl), mean(H), mean(diff.exp() - 1 - diff), mean(((r < 0.8) | (r > 1.2)).float())]
    stats = torch.stack([parts[0] + 0.5 * parts[1] - 0.01 * parts[2], *parts])
    dl = 0.01 * p * (lp + H[:, None]) - g[:, None] * p
    dl.scatter_add_(1, at, g[:, None])
    scale = w / total
    return stats, (dl * scale[:, None]).to(s.logits.dtype), 0.5 * dv * scale


def _plain_adamw(s):
    g = s.grad.float()
    if s.max_norm > 0:
        norm = g.square().sum().sqrt()
        g = g * (s.max_norm / (norm + 1e-6)).clamp(max=1.0)
    s.step += 1
    b1, b2 = s.betas
    m, v = (s.m, s.v) if s.bits == 32 else (_stands(s.m_code.float(), 2, 127, s.m_scale),
                                            _stands(s.v_code.float(), 4, 255, s.v_scale))
    m = b1 * m + (1 - b1) * g
    v = b2 * v + ((1 - b2) * g) * g
    den = v.sqrt() * (1 / math.sqrt(1 - b2 ** s.step)) + s.eps
    p = s.param.float() * (1 - s.lr * s.decay) - (s.lr / (1 - b1 ** s.step)) * (m / den)
    s.param.copy_(p)
    if s.bits == 8:
        qm, s.m_scale = _levels(m, 2, 127)
        qv, s.v_scale = _levels(v, 4, 255)
        s.m_code, s.v_code = qm.to(torch.int8), qv.to(torch.uint8)
        m, v = _stands(qm, 2, 127, s.m_scale), _stands(qv, 4, 255, s.v_scale)
    s.m.copy_(m)
    s.v.copy_(v)
    return s.param, s.m, s.v


def run(s):
    if not own:
        if s.op == "sample":
            return _plain_sample(s.logits, s.uniform, s.mask, **s.settings)
        return _plain_loss(s) if s.op == "loss" else _plain_adamw(s)
    from paper_2607_26005_amd import policy
    if s.op == "sample":
        return policy.sample_actions(s.logits, s.uniform, mask=s.mask, **s.settings)
    if s.op == "loss":
        return policy.policy_gradient(s.logits, s.values, s.actions, s.old_logp, s.advantages, s.returns,
                                      old_values=s.old_values, weights=s.weights, mask=s.mask, clip=0.2,
                                      value_clip=s.value_clip, value_coef=0.5, entropy_coef=0.01,
                                      normalize=s.normalize)
    s.opt.step(grads=s.grads)
    if s.bits == 8:   # what the 8-bit moments stand for
        s.opt.moments(out=s.moments)
    return s.param, s.m, s.v


def work(case):
    size = {"f32": 4, "bf16": 2, "f16": 2}
    if case["op"] == "adamw":
        n = sum(_sizes(case))
        moments = 16 if case["bits"] == 32 else 4 + 16 / _BLOCK + 8   # in and out; 8 bits: and what they stand for
        return {"bytes": n * (2 * size[case["dtype"]] + size[case["grad_dtype"]] + moments), "flops": 16 * n}
    N, NA = case["rows"], case["rows"] * case["actions"]
    logits = NA * (size[case["dtype"]] + (1 if case["mask"] else 0))
    if case["op"] == "sample":
        return {"bytes": logits + N * (16 + (16 if case["per_row"] else 0)), "flops": 4 * NA}
    return {"bytes": logits + NA * size[case["dtype"]] + N * (4 * 6 + 8 + (8 if case["options"] else 0)),
            "flops": 10 * NA}


# ---------------------------------------------------------------------------
# 64-bit references
# ---------------------------------------------------------------------------

def _exact_sample(s):
    N, A = s.logits.shape
    col = lambda k: torch.as_tensor(s.settings[k], device="cuda").double().expand(N)[:, None]
    z = s.logits.double() / col("temperature")
    if s.mask is not None:
        z = torch.where(s.mask, z, -math.inf)
    p = z.softmax(1)
    sp, order = p.sort(dim=1, descending=True, stable=True)
    k = col("top_k")
    keep = (torch.arange(A, device="cuda") < k) | (k <= 0)
    sp = torch.where(keep, sp, 0.0)
    sp = sp / sp.sum(1, keepdim=True)
    before = sp.cumsum(1) - sp
    keep = keep & ((before < col("top_p")) | (col("top_p") >= 1)) & (sp >= col("min_p") * sp[:, :1])
    q = torch.zeros_like(p).scatter_(1, order, torch.where(keep, sp, 0.0))
    q = q / q.sum(1, keepdim=True)
    action = (q.cumsum(1) <= s.uniform.double()[:, None]).sum(1, keepdim=True).clamp(max=A - 1)
    return None, q.gather(1, action)[:, 0].log()   # (the action itself is a whole number)


def _exact_loss(s):
    # by autograd, from the loss alone
    z = s.logits.double().detach().requires_grad_()
    v = s.values.double().detach().requires_grad_()
    w = torch.ones_like(v) if s.weights is None else s.weights.double()
    avg = lambda t: (w * t).sum() / w.sum()
    adv = s.advantages.double()
    if s.normalize:
        adv = (adv - avg(adv)) / (avg((adv - avg(adv)) ** 2).sqrt() + 1e-8)
    masked = z if s.mask is None else z.masked_fill(~s.mask, -1e300)
    logp = masked.log_softmax(1)
    diff = logp.gather(1, s.actions[:, None])[:, 0] - s.old_logp.double()
    ratio = diff.exp()
    pg = avg(-torch.min(ratio * adv, ratio.clamp(0.8, 1.2) * adv))
    R = s.returns.double()
    vl = (v - R) ** 2
    if s.value_clip > 0:
        old = s.old_values.double()
        vl = torch.max(vl, (old + (v - old).clamp(-s.value_clip, s.value_clip) - R) ** 2)
    vl = avg(0.5 * vl)
    H = avg(-(logp.exp() * logp.clamp_min(-1e4)).sum(1))
    loss = pg + 0.5 * vl - 0.01 * H
    dz, dv = torch.autograd.grad(loss, (z, v))
    kl, cut = avg(ratio - 1 - diff), avg(((ratio - 1).abs() > 0.2).double())
    return torch.stack([loss, pg, vl, H, kl, cut]).detach(), dz, dv


def _exact_adamw(s):
    d = lambda t: t.double()
    g, (b1, b2), t = d(s.grad), s.betas, s.step + 1
    if s.max_norm > 0:
        g = g * min(1.0, s.max_norm / (float(g.norm()) + 1e-6))
    m, v = d(s.m), d(s.v)
    if s.bits == 8:
        block = lambda c, sc: (c.view(-1, _BLOCK) * d(sc)[:, None]).view(-1)
        cm, cv = d(s.m_code) / 127, d(s.v_code) / 255
        m, v = block(cm * cm.abs(), s.m_scale), block(cv ** 4, s.v_scale)
    m = b1 * m + (1 - b1) * g
    v = b2 * v + (1 - b2) * g * g
    p = d(s.param) * (1 - s.lr * s.decay)
    p = p - s.lr * (m / (1 - b1 ** t)) / ((v / (1 - b2 ** t)).sqrt() + s.eps)
    if s.bits == 8:
        mb, vb = m.view(-1, _BLOCK), v.view(-1, _BLOCK)
        top = lambda x: x.abs().amax(1, keepdim=True).clamp_min(1e-300)
        qm = ((mb.abs() / top(mb)) ** 0.5 * 127).round() / 127
        qv = ((vb / top(vb)) ** 0.25 * 255).round()
        qv = torch.where(vb > 0, qv.clamp_min(1), qv) / 255
        m, v = (qm * qm * mb.sign() * top(mb)).view(-1), (qv ** 4 * top(vb)).view(-1)
    return p, m, v


def exact(case, seed):
    s = prepare(case, seed)
    return {"sample": _exact_sample, "loss": _exact_loss, "adamw": _exact_adamw}[s.op](s)
