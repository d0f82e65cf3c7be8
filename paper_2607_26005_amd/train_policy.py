"""A small training loop that runs the whole path on the device: views are rendered,
encoded and turned into actions, the agents step, and the policy learns from what
happened.

The paper trains its perspective policy by clipped policy optimisation in the process
that renders for it (Sec. 3.3; App. A.3: clip 0.2, discount 0.999, lambda 0.95,
advantages normalised per minibatch, AdamW at 5e-4, 12 motions of 4 x 3 kinds on a
shared trunk of four layers of 512).  This is that loop in the small, on the synthetic
worlds of `scenegen` and with a reward of its own (keep moving, keep straight): a
pattern for a trainer, not a reproduction of the paper's results.

With --memory the policy remembers the steps of an episode (memory.MemoryLayer): it acts
one step at a time on states that stay on the device and learns from whole rollouts.  With
--prefer it also learns from pairs of agents, of which the one with the larger return over an
episode's steps is preferred in them.

    python -m paper_2607_26005_amd.train_policy --iterations 4 --bits 8
    python -m paper_2607_26005_amd.train_policy --memory 2 --act-bits 8 --prefer 0.1
"""
from __future__ import annotations

import argparse

import torch
import torch.nn as nn

from paper_2607_26005_amd import memory, pictura, policy, scenegen as sg
from paper_2607_26005_amd.encoder import ViewEncoder

ACCELERATIONS = (-3.0, -1.0, 0.0, 2.0)   # m/s^2
STEERING = (-0.2, 0.0, 0.2)              # radians
ACTIONS = len(ACCELERATIONS) * len(STEERING)


class ActorCritic(nn.Module):
    """Views of an ego's cameras -> [egos, ACTIONS + 1]: the motions' logits, then the value."""

    def __init__(self, cams: int = 4, width: int = 512, layers: int = 0):
        super().__init__()
        self.encoder = ViewEncoder(cams=cams)
        trunk, n = [], cams * self.encoder.width
        for _ in range(4):
            trunk += [nn.Linear(n, width), nn.GELU()]
            n = width
        self.trunk = nn.Sequential(*trunk)
        self.head = nn.Linear(width, ACTIONS + 1)
        self.memory = nn.ModuleList(memory.MemoryLayer(width) for _ in range(layers))
        self.norm = nn.Parameter(torch.ones(width)) if layers else None

    def forward(self, cls: torch.Tensor, depth: torch.Tensor) -> torch.Tensor:
        return self.head(self.trunk(self.encoder(cls, depth)))

    def sequence(self, seen, states=None, resets=None) -> torch.Tensor:
        """Views of several steps -> [egos, steps, ACTIONS + 1].  states: what each layer
        remembers before the first; resets [egos, steps]: where an episode begins."""
        x = torch.stack([self.trunk(self.encoder(*views)) for views in seen], 1)
        residual = None
        for i, layer in enumerate(self.memory):
            x, residual, _ = layer(x, residual, None if states is None else states[i], resets)
        return self.head(x if residual is None else memory.rms_norm(x, self.norm, residual)[0])

    @torch.no_grad()
    def act(self, cls: torch.Tensor, depth: torch.Tensor, states, resets=None, codes=None) -> torch.Tensor:
        """One step of the same on `states` (one a layer, replaced) -> [egos, ACTIONS + 1].
        codes: each layer's `quantized` weights, for products in 8 bits."""
        x, residual = self.trunk(self.encoder(cls, depth)), None
        for i, layer in enumerate(self.memory):
            x, residual = layer.step(x, residual, states[i], resets, None if codes is None else codes[i])
        return self.head(x if residual is None else memory.rms_norm(x, self.norm, residual)[0])


def controls(actions: torch.Tensor):
    """(steer, accel) of motion indices; an agent that drew none (-1) coasts straight on."""
    accel = torch.tensor(ACCELERATIONS, device=actions.device)
    steer = torch.tensor(STEERING, device=actions.device)
    a = torch.where(actions < 0, ACTIONS, actions)
    table = torch.cat([torch.stack([steer.repeat(len(ACCELERATIONS)), accel.repeat_interleave(len(STEERING))]),
                       torch.zeros(2, 1, device=actions.device)], 1)
    return table[0][a].contiguous(), table[1][a].contiguous()


def advantages(rewards, values, last_value, gamma: float = 0.999, lam: float = 0.95):
    """Generalised advantage estimates and returns of [steps, agents] rewards and values."""
    out, run = torch.empty_like(rewards), torch.zeros_like(last_value)
    for t in reversed(range(len(rewards))):
        after = values[t + 1] if t + 1 < len(values) else last_value
        run = rewards[t] + gamma * after - values[t] + gamma * lam * run
        out[t] = run
    return out, out + values


def preferred(returns: torch.Tensor, resets: torch.Tensor):
    """Pairs for the preference loss from [agents, steps] of a rollout, of every episode in it its
    own: (rows of the [agents * steps] decisions, one sequence behind the other; offsets).  The
    agent with the larger return over an episode's steps comes first.  All agents' episodes begin
    together."""
    n, steps = returns.shape
    half, began = n // 2, resets[:1].any(0).tolist()
    starts = [t for t in range(steps) if t == 0 or began[t]]
    rows, lengths = [], [0]
    for a, b in zip(starts, starts[1:] + [steps]):
        order = returns[:, a].argsort(descending=True)
        pairs = torch.stack([order[:half], order[n - half:]], 1).reshape(-1, 1)
        rows.append((pairs * steps + torch.arange(a, b, device=returns.device)).reshape(-1))
        lengths += [b - a] * (2 * half)
    return torch.cat(rows), torch.tensor(lengths, device=returns.device).cumsum(0)


class Trainer:
    """`worlds` worlds of the paper's rig (32 agents each, four cameras at 96x54)."""

    def __init__(self, worlds: int = 2, bits: int = 32, seed: int = 0, device: int = 0, layers: int = 0, act_bits: int = 32,
                 episode: int = 0):
        self.workload = sg.make_config(6, num_worlds=worlds)
        self.rig = self.workload.rig
        self.renderer = pictura.Renderer(device)
        self.renderer.upload(self.workload.scene, self.workload.cell_size)
        self.agents = pictura.DeviceAgents.from_host(self.workload.agents, f"cuda:{device}")
        torch.manual_seed(seed)
        self.net = ActorCritic(cams=self.rig.num_cams, layers=layers).to(f"cuda:{device}")
        self.opt = policy.AdamW(self.net.parameters(), lr=5e-4, weight_decay=0.01, bits=bits, max_norm=0.5)
        self.random = torch.Generator(f"cuda:{device}").manual_seed(seed)
        # with a memory: what is remembered, steps since the episode began, and where it began
        n = self.agents.x.numel()
        self.states = [torch.zeros(n, layer.width, device=f"cuda:{device}") for layer in self.net.memory]
        self.act_bits, self.episode, self.age = act_bits, episode, 0
        self.start = {k: getattr(self.agents, k).clone() for k in ("x", "y", "psi", "speed", "cos_h", "sin_h")}

    def close(self):
        self.renderer.close_checked()

    def rollout(self, steps: int):
        """`steps` decisions of every agent: what was seen, done and earned."""
        n = self.agents.x.numel()
        seen, did = [], []
        with torch.no_grad():
            for _ in range(steps + 1):
                cls, depth = self.renderer.render(self.agents, self.rig)
                out = self.net(cls, depth)
                logits, values = out[:, :ACTIONS], out[:, ACTIONS]
                if len(seen) == steps:
                    break
                u = torch.rand(n, device=out.device, generator=self.random)
                actions, logp = policy.sample_actions(logits, u)
                steer, accel = controls(actions)
                self.renderer.agents_step(self.agents, steer, accel)
                seen.append((cls, depth))
                did.append((actions, logp, values.clone(), 0.1 * self.agents.speed - steer.abs()))
        actions, logp, old_values, rewards = (torch.stack(t) for t in zip(*did))
        adv, returns = advantages(rewards, old_values, values)
        return seen, actions, logp, old_values, adv, returns

    def _begin(self):
        """Whether an episode begins with this step, for every agent; all are put back then."""
        begins = self.age == 0
        if begins:
            for k, v in self.start.items():
                getattr(self.agents, k).copy_(v)
        self.age += 1
        if self.episode and self.age == self.episode:
            self.age = 0
        return torch.full_like(self.agents.x, begins, dtype=torch.bool)

    @torch.no_grad()
    def remembered_rollout(self, steps: int):
        """As rollout, by the policy that remembers: (views, resets [agents, steps], states
        before the first step, actions, log-probabilities, values, advantages, returns), the
        last five [agents, steps].  No value is carried over the end of an episode."""
        n = self.agents.x.numel()
        codes = [layer.quantized() for layer in self.net.memory] if self.act_bits == 8 else None
        before, seen, did = [s.clone() for s in self.states], [], []
        for _ in range(steps):
            began = self._begin()
            cls, depth = self.renderer.render(self.agents, self.rig)
            out = self.net.act(cls, depth, self.states, began, codes)
            actions, logp = policy.sample_actions(out[:, :ACTIONS], torch.rand(n, device=out.device, generator=self.random))
            steer, accel = controls(actions)
            self.renderer.agents_step(self.agents, steer, accel)
            seen.append((cls, depth))
            did.append((began, actions, logp, out[:, ACTIONS].clone(), 0.1 * self.agents.speed - steer.abs()))
        resets, actions, logp, values, rewards = (torch.stack(t) for t in zip(*did))
        # each episode's own estimates; the last one goes on from what the next step would be worth
        adv, returns = torch.empty_like(rewards), torch.empty_like(rewards)
        starts = [t for t in range(1, steps) if self.episode and bool(resets[t, 0])]
        for a, b in zip([0] + starts, starts + [steps]):
            after = torch.zeros_like(values[0])
            if b == steps and self.age != 0:   # (the states are not moved by looking ahead)
                cls, depth = self.renderer.render(self.agents, self.rig)
                after = self.net.act(cls, depth, [s.clone() for s in self.states], None, codes)[:, ACTIONS]
            adv[a:b], returns[a:b] = advantages(rewards[a:b], values[a:b], after)
        return (seen, resets.t(), before, *(t.t().contiguous() for t in (actions, logp, values, adv, returns)))

    def remembered_update(self, batch, epochs: int = 2, prefer: float = 0.0):
        """The whole rollout as a minibatch, once an epoch; with prefer also that much of the
        preference loss over pairs of agents, episode by episode.  Returns the last statistics of both."""
        seen, resets, before, actions, logp, values, adv, returns = batch
        n, steps = actions.shape
        flat = lambda t: t.reshape(-1)
        if prefer:
            rows_of, offsets = preferred(returns, resets)
            did, before_logp = flat(actions)[rows_of], flat(logp)[rows_of]
        stats = liked = None
        for _ in range(epochs):
            out = self.net.sequence(seen, before, resets)
            rows = out.reshape(n * steps, ACTIONS + 1)
            loss, stats = policy.policy_loss(rows[:, :ACTIONS], rows[:, ACTIONS], flat(actions), flat(logp), flat(adv),
                                             flat(returns), old_values=flat(values), clip=0.2, value_clip=0.2, normalize=True)
            if prefer:
                other, liked, _ = policy.preference_loss(rows[rows_of, :ACTIONS], did, offsets, before_logp)
                loss = loss + prefer * other
            self.opt.zero_grad()
            loss.backward()
            self.opt.step()
        return stats, liked

    def update(self, batch, epochs: int = 2):
        """Every step's views once an epoch as a minibatch; returns the last statistics."""
        seen, *rest = batch
        stats = None
        for _ in range(epochs):
            for (cls, depth), actions, logp, old_values, adv, returns in zip(seen, *rest):
                out = self.net(cls, depth)
                loss, stats = policy.policy_loss(out[:, :ACTIONS], out[:, ACTIONS], actions, logp, adv, returns,
                                                 old_values=old_values, clip=0.2, value_clip=0.2, normalize=True)
                self.opt.zero_grad()
                loss.backward()
                self.opt.step()
        return stats


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--worlds", type=int, default=2)
    ap.add_argument("--steps", type=int, default=8)
    ap.add_argument("--iterations", type=int, default=4)
    ap.add_argument("--bits", type=int, default=32, choices=(32, 8), help="of the optimizer's moments")
    ap.add_argument("--memory", type=int, default=0, metavar="LAYERS", help="layers with a memory over the episode's steps")
    ap.add_argument("--episode", type=int, default=0, help="steps of an episode (with --memory; 0: it never ends)")
    ap.add_argument("--act-bits", type=int, default=32, choices=(32, 8), help="of the memory's projections when acting")
    ap.add_argument("--prefer", type=float, default=0.0, metavar="WEIGHT", help="of the preference loss (with --memory)")
    a = ap.parse_args()
    if not a.memory and (a.prefer or a.episode or a.act_bits == 8):
        ap.error("--prefer, --episode and --act-bits 8 go with --memory")
    t = Trainer(a.worlds, bits=a.bits, layers=a.memory, act_bits=a.act_bits, episode=a.episode)
    try:
        for i in range(a.iterations):
            if a.memory:
                batch = t.remembered_rollout(a.steps)
                values, liked = t.remembered_update(batch, prefer=a.prefer)
                stats = dict(zip(policy.POLICY_STATS, values.tolist()))
                if liked is not None:
                    stats.update(("preference " + k, v) for k, v in zip(policy.PREFERENCE_STATS, liked.tolist()))
                earned = batch[7]
            else:
                batch = t.rollout(a.steps)
                stats = dict(zip(policy.POLICY_STATS, t.update(batch).tolist()))
                earned = batch[5]
            print(f"iteration {i}: return {earned.mean().item():+.3f}, " +
                  ", ".join(f"{k} {v:.4f}" for k, v in stats.items()) + f", gradient {t.opt.grad_norm.item():.3f}", flush=True)
    finally:
        t.close()


if __name__ == "__main__":
    main()
