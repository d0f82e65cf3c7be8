"""A small training loop that runs the whole path on the device: views are rendered,
encoded and turned into actions, the agents step, and the policy learns from what
happened.

The paper trains its perspective policy by clipped policy optimisation in the process
that renders for it (Sec. 3.3; App. A.3: clip 0.2, discount 0.999, lambda 0.95,
advantages normalised per minibatch, AdamW at 5e-4, 12 motions of 4 x 3 kinds on a
shared trunk of four layers of 512).  This is that loop in the small, on the synthetic
worlds of `scenegen` and with a reward of its own (keep moving, keep straight): a
pattern for a trainer, not a reproduction of the paper's results.

    python -m paper_2607_26005_amd.train_policy --iterations 4 --bits 8
"""
from __future__ import annotations

import argparse

import torch
import torch.nn as nn

from paper_2607_26005_amd import pictura, policy, scenegen as sg
from paper_2607_26005_amd.encoder import ViewEncoder

ACCELERATIONS = (-3.0, -1.0, 0.0, 2.0)   # m/s^2
STEERING = (-0.2, 0.0, 0.2)              # radians
ACTIONS = len(ACCELERATIONS) * len(STEERING)


class ActorCritic(nn.Module):
    """Views of an ego's cameras -> [egos, ACTIONS + 1]: the motions' logits, then the value."""

    def __init__(self, cams: int = 4, width: int = 512):
        super().__init__()
        self.encoder = ViewEncoder(cams=cams)
        layers, n = [], cams * self.encoder.width
        for _ in range(4):
            layers += [nn.Linear(n, width), nn.GELU()]
            n = width
        self.trunk = nn.Sequential(*layers)
        self.head = nn.Linear(width, ACTIONS + 1)

    def forward(self, cls: torch.Tensor, depth: torch.Tensor) -> torch.Tensor:
        return self.head(self.trunk(self.encoder(cls, depth)))


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


class Trainer:
    """`worlds` worlds of the paper's rig (32 agents each, four cameras at 96x54)."""

    def __init__(self, worlds: int = 2, bits: int = 32, seed: int = 0, device: int = 0):
        self.workload = sg.make_config(6, num_worlds=worlds)
        self.rig = self.workload.rig
        self.renderer = pictura.Renderer(device)
        self.renderer.upload(self.workload.scene, self.workload.cell_size)
        self.agents = pictura.DeviceAgents.from_host(self.workload.agents, f"cuda:{device}")
        torch.manual_seed(seed)
        self.net = ActorCritic(cams=self.rig.num_cams).to(f"cuda:{device}")
        self.opt = policy.AdamW(self.net.parameters(), lr=5e-4, weight_decay=0.01, bits=bits, max_norm=0.5)
        self.random = torch.Generator(f"cuda:{device}").manual_seed(seed)

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
    a = ap.parse_args()
    t = Trainer(a.worlds, bits=a.bits)
    try:
        for i in range(a.iterations):
            batch = t.rollout(a.steps)
            stats = dict(zip(policy.POLICY_STATS, t.update(batch).tolist()))
            print(f"iteration {i}: return {batch[5].mean().item():+.3f}, " +
                  ", ".join(f"{k} {v:.4f}" for k, v in stats.items()) + f", gradient {t.opt.grad_norm.item():.3f}", flush=True)
    finally:
        t.close()


if __name__ == "__main__":
    main()
