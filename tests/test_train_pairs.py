"""The pairs that train_policy --prefer learns from: what is preferred is decided by the steps that
the loss then compares (host tensors and stand-ins for the kernels; no GPU needed)."""
import types

import pytest
import torch

from paper_2607_26005_amd import policy, train_policy as tp


def _compared(monkeypatch, returns, resets):
    """[(agent, first step, steps beyond the last)] of the sequences that the loss is given."""
    n, steps = returns.shape
    row = torch.arange(n * steps, dtype=torch.float32).reshape(n, steps, 1)
    net = types.SimpleNamespace(sequence=lambda seen, states, resets: row.expand(n, steps, tp.ACTIONS + 1).clone().requires_grad_())
    opt = types.SimpleNamespace(zero_grad=lambda: None, step=lambda: None)
    given = []

    def loss(logits, actions, offsets, ref_logp, **k):
        assert torch.equal(logits[:, 0], actions.float()) and torch.equal(logits[:, 0], ref_logp)
        given.append((logits[:, 0].long(), offsets.tolist()))
        return logits.sum() * 0, torch.zeros(4), None

    monkeypatch.setattr(policy, "policy_loss", lambda rows, *a, **k: (rows.sum() * 0, torch.zeros(6)))
    monkeypatch.setattr(policy, "preference_loss", loss)
    flat = row[..., 0]
    batch = (None, resets, None, flat.long(), flat, flat, flat, returns)
    tp.Trainer.remembered_update(types.SimpleNamespace(net=net, opt=opt), batch, epochs=1, prefer=0.1)
    (rows, offsets), = given
    assert offsets[0] == 0 and offsets[-1] == len(rows) and len(offsets) % 2 == 1
    found = []
    for a, b in zip(offsets, offsets[1:]):
        agents, at = rows[a:b] // steps, rows[a:b] % steps
        assert b > a and (agents == agents[0]).all() and torch.equal(at, torch.arange(at[0], at[0] + b - a))
        found.append((agents[0].item(), at[0].item(), at[0].item() + b - a))
    return found


@pytest.mark.parametrize("n", [1, 2, 7, 8])
@pytest.mark.parametrize("starts", [[], [3], [0], [0, 3, 6], [1, 2, 4]])
def test_pairs_are_preferred_by_the_steps_they_span(monkeypatch, n, starts):
    steps = 7
    returns = torch.randn(n, steps, generator=torch.Generator().manual_seed(n))
    resets = torch.zeros(n, steps, dtype=torch.bool)
    resets[:, starts] = True
    found = _compared(monkeypatch, returns, resets)
    ends = sorted({0, *starts}) + [steps]
    # every episode has its own pairs, of agents that stand in one each
    assert len(found) == (len(ends) - 1) * 2 * (n // 2)
    for a, b in zip(ends, ends[1:]):
        here = [f for f in found if f[1] == a]
        assert len({f[0] for f in here}) == len(here) == 2 * (n // 2) and all(f[2] == b for f in here)
    for better, other in zip(found[::2], found[1::2]):
        assert better[1:] == other[1:]
        assert returns[better[0], better[1]] > returns[other[0], other[1]]   # the return of just these steps
