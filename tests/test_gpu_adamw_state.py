"""AdamW as a program keeps it: its groups, copies and saved states."""
import copy
import pickle

import pytest
import torch

from paper_2608_10805_amd import autograd, optim

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
LR = 1e-2
LAST = torch.channels_last


def image_kernel(seed=0, shape=(8, 6, 3, 3), dtype=torch.float32):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return torch.nn.Parameter(torch.randn(shape, generator=g, device=DEV).to(dtype))


def some_grad(p, t):
    g = torch.Generator(device=DEV).manual_seed(100 + t)
    return torch.randn(p.shape, generator=g, device=DEV).to(p.dtype) * 1e-2


def both_paths(monkeypatch, native):
    """The native host path, or Python alone."""
    if not native:
        monkeypatch.setattr(autograd, "load_block", lambda x: False)


def take(opt, ps, t):
    for p in ps:
        p.grad = torch.empty_like(p, requires_grad=False).copy_(some_grad(p, t))
    opt.step()


@pytest.mark.parametrize("native", [True, False])
def test_parameters_of_a_changed_group_are_refused(native, monkeypatch):
    """The moments belong to the parameters that the group was added with, in their order."""
    both_paths(monkeypatch, native)
    ps = [image_kernel(i, (8, 9)) for i in range(3)]
    opt = optim.AdamW(ps, lr=LR)
    take(opt, ps, 0)
    kept = [p.detach().clone() for p in ps]
    group = opt.param_groups[0]
    for changed in (ps[1:], [ps[1], ps[0], ps[2]], ps + [image_kernel(7)], ps[:2] + [image_kernel(8, (8, 9))]):
        for p in changed:
            p.grad = some_grad(p, 1)
        group["params"] = changed
        with pytest.raises(ValueError, match="parameters"):
            opt.step()
        assert all(torch.equal(p.detach(), k) for p, k in zip(ps, kept))
    group["params"] = list(ps)
    opt.step()
    assert [int(opt.state[p]["step"]) for p in ps] == [2, 2, 2]


@pytest.mark.parametrize("bits", [8, 32])
@pytest.mark.parametrize("how", ["deepcopy", "pickle"])
def test_copies_of_an_optimizer_go_on_by_themselves(bits, how):
    """A copy has parameters, moments, steps and a seed of its own, and steps as the first one does."""
    ps = [image_kernel(), image_kernel(1, (70, 9), torch.bfloat16), image_kernel(2, (1,))]
    ps[0].data = ps[0].data.to(memory_format=LAST)
    opt = optim.AdamW([{"params": ps[:1], "lr": 0.1}, {"params": ps[1:]}], lr=LR, state_bits=bits, seed=6)
    take(opt, ps, 0)
    other = copy.deepcopy(opt) if how == "deepcopy" else pickle.loads(pickle.dumps(opt))
    qs = [p for g in other.param_groups for p in g["params"]]
    kept = [q.detach().clone() for q in qs]
    assert all(torch.equal(p.detach(), q) for p, q in zip(ps, kept))
    take(opt, ps, 1)
    assert all(torch.equal(q.detach(), k) for q, k in zip(qs, kept))  # its own memory
    assert all(int(other.state[q]["step"]) == 1 for q in qs)
    take(other, qs, 1)
    assert all(torch.equal(p.detach(), q.detach()) for p, q in zip(ps, qs))
    assert all(torch.equal(a, b) for x, y in zip(opt.moments(), other.moments()) for a, b in zip(x, y))
    assert other.param_groups[0]["lr"] == 0.1 and other.state_bits == bits and other.seed == 6
    other.add_param_group({"params": [image_kernel(3)]})
    other.load_state_dict(copy.deepcopy(other.state_dict()))


def test_a_copy_keeps_the_order_that_8_bit_moments_are_in():
    """Also where a parameter has left it since the last step: both optimizers refuse the next one."""
    p = image_kernel()
    opt = optim.AdamW([p], lr=LR, state_bits=8)
    take(opt, [p], 0)
    p.data = p.data.to(memory_format=LAST)
    other = copy.deepcopy(opt)
    q = other.param_groups[0]["params"][0]
    for o, t in ((opt, p), (other, q)):
        with pytest.raises(ValueError, match="order"):
            take(o, [t], 1)
        t.data = t.data.contiguous()
        take(o, [t], 1)
    assert torch.equal(p.detach(), q.detach())


def test_a_resumed_run_rounds_as_the_first_one_would_have(tmp_path):
    """The seed is part of the state, also through a file that is read without running anything from it."""
    p = image_kernel()
    opt = optim.AdamW([p], lr=LR, state_bits=8, seed=11)
    take(opt, [p], 0)
    torch.save(opt.state_dict(), tmp_path / "state.pt")
    q = torch.nn.Parameter(p.detach().clone())
    other = optim.AdamW([q], lr=0.5, state_bits=8, seed=12)
    other.load_state_dict(torch.load(tmp_path / "state.pt", weights_only=True))
    for t in (1, 2):
        take(opt, [p], t)
        take(other, [q], t)
    assert torch.equal(p.detach(), q.detach())
    assert all(torch.equal(a, b) for a, b in zip(opt.moments()[0], other.moments()[0]))


def test_hooks_around_loading_a_state():
    p, q = image_kernel(), image_kernel()
    a, b = (optim.AdamW([t], lr=LR) for t in (p, q))
    take(a, [p], 0)
    seen = []

    def before(opt, state):
        seen.append("before")
        assert opt is b and int(b.state[q]["step"]) == 0
        return {**state, "param_groups": [{**g, "lr": 0.25} for g in state["param_groups"]]}

    def after(opt):
        seen.append("after")
        assert opt is b and int(b.state[q]["step"]) == 1

    b.register_load_state_dict_pre_hook(before)
    b.register_load_state_dict_post_hook(after)
    b.load_state_dict(copy.deepcopy(a.state_dict()))
    assert seen == ["before", "after"] and b.param_groups[0]["lr"] == 0.25 and a.param_groups[0]["lr"] == LR


@pytest.mark.parametrize("bits", [8, 32])
def test_an_empty_group_stays_on_the_native_path(bits, monkeypatch):
    """It neither sends the others through Python nor changes their random bits, and its moments are empty."""
    runs = []
    for native in (True, False):
        ps = [image_kernel(), image_kernel(1)]
        opt = optim.AdamW([{"params": ps[:1]}, {"params": []}, {"params": ps[1:]}], lr=LR, state_bits=bits)
        if native:
            monkeypatch.setattr(opt, "_step", lambda scale: pytest.fail("left to Python"))
        else:
            opt._native = [None] * 3
        take(opt, ps, 0)
        take(opt, ps, 1)
        m, v = opt.moments()[1]
        assert m.numel() == v.numel() == 0
        assert m.dtype == v.dtype == (torch.bfloat16 if bits == 8 else torch.float32)
        runs.append([p.detach().clone() for p in ps])
    assert all(torch.equal(a, b) for a, b in zip(*runs))


@pytest.mark.parametrize("native", [True, False])
@pytest.mark.parametrize("bits", [8, 32])
def test_parameters_of_no_elements(native, bits, monkeypatch):
    """By themselves and beside others, with gradients."""
    both_paths(monkeypatch, native)
    none, some = torch.nn.Parameter(torch.empty(0, 3, device=DEV)), image_kernel()
    alone = optim.AdamW([none], state_bits=bits)
    mixed = optim.AdamW([{"params": [none]}, {"params": [some, none.detach()]}], state_bits=bits)
    none.grad = torch.empty(0, 3, device=DEV)
    alone.step()
    assert int(alone.state[none]["step"]) == 1
    kept = some.detach().clone()
    take(mixed, [some], 0)
    assert not torch.equal(some.detach(), kept)


def test_a_group_that_cannot_be_added_is_not_there():
    """Whatever was wrong with it."""
    p = image_kernel()
    opt = optim.AdamW([p], lr=LR)
    for bad, error in (({"params": [image_kernel(1)], "lr": None}, TypeError),
                       ({"params": [image_kernel(2)], "betas": 0.9}, TypeError),
                       ({"params": [image_kernel(3)], "eps": -1.0}, ValueError)):
        with pytest.raises(error):
            opt.add_param_group(bad)
        assert len(opt.param_groups) == len(opt._buffers) == len(opt._native) == 1
    take(opt, [p], 0)
    opt.add_param_group({"params": [image_kernel(4)]})
    assert len(opt.param_groups) == len(opt._buffers) == 2
