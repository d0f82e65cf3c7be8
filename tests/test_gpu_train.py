"""The training loop that runs rendering, encoding, drawing actions, the policy loss and
the optimizer together on the device (paper_2607_26005_amd/train_policy.py)."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits", [32, 8])
def test_policy_learns_from_a_rollout(bits):
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no HIP device")
    from paper_2607_26005_amd import policy, train_policy as tp
    t = tp.Trainer(worlds=1, bits=bits, seed=1)
    try:
        before = [p.detach().clone() for p in t.net.parameters()]
        batch = t.rollout(4)
        seen, actions, logp, values, adv, returns = batch
        n = t.agents.x.numel()
        assert len(seen) == 4 and actions.shape == logp.shape == values.shape == adv.shape == (4, n)
        assert ((actions >= 0) & (actions < tp.ACTIONS)).all() and (logp < 0).all()
        # a fresh head is close to even: the drawn log-probabilities are its own
        with torch.no_grad():
            out = t.net(*seen[0])
            want = out[:, :tp.ACTIONS].log_softmax(1).gather(1, actions[0][:, None])[:, 0]
        assert torch.allclose(logp[0], want, atol=1e-4)
        # the same minibatch again and again: the loss that is followed downhill falls
        one = [x[:1] for x in batch]
        stats = [dict(zip(policy.POLICY_STATS, t.update(one, epochs=1).tolist())) for _ in range(20)]
        assert stats[-1]["loss"] < stats[0]["loss"] and stats[-1]["policy_loss"] < stats[0]["policy_loss"], (stats[0], stats[-1])
        assert abs(stats[0]["approx_kl"]) < 1e-5 < stats[-1]["approx_kl"]   # the policy moved away from the one that acted
        t.update(batch)
        assert all(torch.isfinite(p).all() for p in t.net.parameters())
        assert all((p != b).any() for p, b in zip(t.net.parameters(), before))
        assert t.opt.grad_norm.isfinite()
    finally:
        t.close()


def test_controls_of_every_action():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no HIP device")
    from paper_2607_26005_amd import train_policy as tp
    steer, accel = tp.controls(torch.arange(-1, tp.ACTIONS, device="cuda"))
    assert steer[0] == 0 and accel[0] == 0
    pairs = {(round(s, 4), round(a, 4)) for s, a in zip(steer[1:].tolist(), accel[1:].tolist())}
    assert pairs == {(s, a) for s in tp.STEERING for a in tp.ACCELERATIONS}
