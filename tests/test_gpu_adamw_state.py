"""AdamW as a program keeps it: its groups, copies and saved states."""
import pytest
import torch

from paper_2608_10805_amd import autograd, optim

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
LR = 1e-2


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
