"""What the optimizer and the loss keep and check around their kernels: host tensors
stand in for device ones, and a launch is recorded, not made (no GPU needed)."""
import copy
import pickle

import pytest
import torch

from paper_2607_26005_amd import pictura, policy


@pytest.fixture
def launches(monkeypatch):
    """The devices of the launches that would have been made."""
    made = []
    monkeypatch.setattr(pictura, "_call", lambda device, fn, *args: made.append(device) or pictura.OK)
    return made


@pytest.fixture
def any_device(monkeypatch):
    monkeypatch.setattr(pictura, "_check_device", lambda t, name, ctx: None)


def _param(*shape, device="cpu"):
    return torch.nn.Parameter(torch.zeros(*shape, device=device))


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("listed", [False, True])
def test_a_step_refuses_host_weights_behind_a_frozen_one(launches, bits, listed):
    # parameter 0 takes no part; parameter 1 is on the host: its address is none for a kernel
    frozen, head = _param(4, device="meta"), _param(4)
    head.grad = torch.ones(4)
    opt = policy.AdamW([frozen, head], bits=bits, max_norm=1.0)
    with pytest.raises(pictura.PicturaError, match="parameter 1: tensor on cpu, expected the HIP device"):
        opt.step(grads=[None, torch.ones(4)] if listed else None)
    assert launches == []


def test_a_step_runs_on_the_device_of_the_weights_that_take_part(launches, any_device):
    frozen, head = _param(4, device="meta"), _param(4)
    head.grad = torch.ones(4)
    policy.AdamW([frozen, head]).step()
    assert launches == [head.device]
    other = _param(4)
    other.grad = torch.ones(4)
    with pytest.raises(pictura.PicturaError, match="parameter 2: on meta, others on cpu"):
        moved = _param(4, device="meta")
        moved.grad = torch.ones(4, device="meta")
        policy.AdamW([frozen, other, moved]).step()
    assert launches == [head.device]


@pytest.mark.parametrize("bits", [32, 8])
def test_a_step_counts_as_a_change_of_the_weights(launches, any_device, bits):
    # as torch's optimizers: a graph that saved the weights before the step is refused after it
    w, still, x = _param(3), _param(3), torch.ones(3, requires_grad=True)
    opt = policy.AdamW([still, w], bits=bits)
    loss = (w * x).sum()
    loss.backward(retain_graph=True)
    before = w._version
    opt.step()
    assert (w._version, still._version) == (before + 1, 0)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        loss.backward()
    opt.step(grads=[torch.ones(3), None])
    assert (w._version, still._version) == (before + 1, 1)
    opt.moments()
    assert (w._version, still._version) == (before + 1, 1)
    with torch.inference_mode():
        p = torch.nn.Parameter(torch.zeros(3))
    policy.AdamW([p]).step(grads=[torch.ones(3)])   # (such a tensor has no version)
    assert len(launches) == 2 + (bits == 8) + 1


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("kept", [{}, {"mine": 1}])
def test_a_state_that_was_read_before_the_first_step_is_begun_by_it(launches, any_device, bits, kept):
    ps = [_param(3), _param(300)]
    opt = policy.AdamW(ps, bits=bits)
    for p in ps:
        opt.state[p].update(kept)                            # reading makes an empty state
    assert opt.moments() == ([], [])
    opt.step(grads=[torch.ones(3), None])
    assert opt.state[ps[0]]["step"] == 1 and opt.state[ps[0]]["exp_avg"].numel() == 3 and opt.state[ps[1]] == kept
    assert [len(m) for m in opt.moments()] == [1, 1]
    opt.step(grads=[torch.ones(3), torch.ones(300)])
    assert [opt.state[p]["step"] for p in ps] == [2, 1]
    assert [len(m) for m in opt.moments()] == [2, 2]
    assert all(opt.state[p].items() >= kept.items() for p in ps)


@pytest.mark.parametrize("bits, max_norm", [(32, None), (8, 0.5)])
@pytest.mark.parametrize("how", [copy.deepcopy, lambda o: pickle.loads(pickle.dumps(o))], ids=["copy", "pickle"])
@pytest.mark.parametrize("stepped", [False, True])
def test_copies_of_an_optimizer_step_as_it_does(launches, any_device, bits, max_norm, how, stepped):
    opt = policy.AdamW([_param(300)], lr=0.25, bits=bits, max_norm=max_norm)
    if stepped:
        opt.step(grads=[torch.ones(300)])
    other = how(opt)
    assert (other.bits, other.max_norm, other.param_groups[0]["lr"]) == (bits, max_norm, 0.25)
    assert (other.grad_norm is None) == (opt.grad_norm is None)
    del launches[:]
    other.step(grads=[torch.ones(300)])
    q = other.param_groups[0]["params"][0]
    assert other.state[q]["step"] == 1 + stepped and opt.param_groups[0]["params"][0] is not q
    assert other.state[q]["exp_avg"].dtype == (torch.float32 if bits == 32 else torch.int8)
    assert len(launches) == 1 + (max_norm is not None)


def test_a_checkpoint_keeps_the_clipping_norm(launches, any_device):
    opt = policy.AdamW([_param(300)], lr=0.25, max_norm=0.5)
    opt.step(grads=[torch.ones(300)])
    held = opt.state_dict()
    for max_norm in (None, 2.0):
        other = policy.AdamW([_param(300)], max_norm=max_norm)
        other.load_state_dict(copy.deepcopy(held))
        assert other.max_norm == 0.5 and other.param_groups[0]["lr"] == 0.25
        # one that does not have it (torch's own, or an earlier one) leaves what the optimizer was made with
        other = policy.AdamW([_param(300)], max_norm=max_norm)
        other.load_state_dict({k: held[k] for k in ("state", "param_groups")})
        assert other.max_norm == max_norm
    off = policy.AdamW([_param(300)], max_norm=2.0)
    off.load_state_dict(policy.AdamW([_param(300)]).state_dict())
    assert off.max_norm is None


def test_hooks_of_a_load_are_heard(launches, any_device):
    source, target = (policy.AdamW([torch.nn.Parameter(torch.zeros(4, dtype=torch.bfloat16))]) for _ in range(2))
    q = target.param_groups[0]["params"][0]
    source.step(grads=[torch.ones(4)])
    held = source.state_dict()
    precise = torch.full((4,), 1 + 2.0 ** -20)               # (no number in bfloat16, which torch would make it)

    def before(opt, d):
        return dict(d, state={0: dict(d["state"][0], exp_avg=precise, step=7)})

    def after(opt):
        assert torch.equal(opt.state[q]["exp_avg"], precise) and opt.state[q]["step"] == 7
        opt.state[q]["step"] = 9

    hooks = target.register_load_state_dict_pre_hook(before), target.register_load_state_dict_post_hook(after)
    target.load_state_dict(held)
    assert target.state[q]["step"] == 9 and torch.equal(target.state[q]["exp_avg"], precise)
    for h in hooks:
        h.remove()
    assert not target._optimizer_load_state_dict_pre_hooks and not target._optimizer_load_state_dict_post_hooks
    target.load_state_dict(held)
    assert target.state[q]["step"] == 1 and torch.equal(target.state[q]["exp_avg"], torch.zeros(4))
    with pytest.raises(ValueError):
        target.load_state_dict({"state": {}, "param_groups": []})
    assert not target._optimizer_load_state_dict_pre_hooks and not target._optimizer_load_state_dict_post_hooks


@pytest.mark.parametrize("name", ["temperature", "top_k", "top_p", "min_p"])
@pytest.mark.parametrize("v", [10 ** 400, -10 ** 400])
def test_sampling_refuses_numbers_beyond_its_types(launches, any_device, name, v):
    n, a = 3, 5
    if name == "top_k":
        policy.sample_actions(torch.zeros(n, a), torch.zeros(n), top_k=v)   # any whole number: cut to what counts
        assert len(launches) == 1
        return
    with pytest.raises(pictura.PicturaError, match=name) as e:
        policy.sample_actions(torch.zeros(n, a), torch.zeros(n), **{name: v})
    assert e.value.status == pictura.EINVAL and launches == []


@pytest.mark.parametrize("name", ["temperature", "clip", "value_clip", "value_coef", "entropy_coef", "denominator"])
@pytest.mark.parametrize("v", [10 ** 400, "much", None])
def test_loss_refuses_numbers_beyond_its_types(launches, any_device, name, v):
    n = 3
    z, i = torch.zeros(n), torch.zeros(n, dtype=torch.int64)
    with pytest.raises(pictura.PicturaError, match=f"{name}: ") as e:
        policy.policy_gradient(torch.zeros(n, 5), z, i, z, z, z, **{name: v})
    assert e.value.status == pictura.EINVAL and launches == []


@pytest.mark.parametrize("name", ["lr", "eps", "weight_decay"])
@pytest.mark.parametrize("v", [10 ** 400, "much"])
def test_steps_refuse_numbers_beyond_their_types(launches, any_device, name, v):
    opt = policy.AdamW([_param(3)])
    opt.param_groups[0][name] = v
    with pytest.raises(pictura.PicturaError, match=f"{name}: ") as e:
        opt.step(grads=[torch.ones(3)])
    assert e.value.status == pictura.EINVAL and launches == []


def test_groups_that_moved_before_a_refused_one_have_counted(launches, any_device, monkeypatch):
    ps = [_param(3) for _ in range(4)]
    opt = policy.AdamW([dict(params=ps[:2]), dict(params=ps[2:])])
    opt.step(grads=[torch.ones(3)] * 4)
    opt.param_groups[1]["betas"] = (0.9, 2.0)
    call = pictura._call                                     # (the entry refuses such a beta before it launches)
    monkeypatch.setattr(pictura, "_call", lambda device, fn, how, *args: pictura.EINVAL
                        if pictura._ADAMW_PACK.unpack(how)[2] == 2.0 else call(device, fn, how, *args))
    with pytest.raises(pictura.PicturaError):
        opt.step(grads=[torch.ones(3), None, torch.ones(3), torch.ones(3)])
    assert [opt.state[p]["step"] for p in ps] == [2, 1, 1, 1] and len(launches) == 3
