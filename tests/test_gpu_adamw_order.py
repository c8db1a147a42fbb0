"""AdamW on parameters whose memory has, or gets, another order than their shape's."""
import copy

import pytest
import torch

from paper_2608_10805_amd import autograd, optim

from tests import _block as ref

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


# ----------------------------------------------------------------------------
# the order of a parameter's memory
# ----------------------------------------------------------------------------

@pytest.mark.parametrize("native", [True, False])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("back", [False, True])
def test_32_bit_moments_follow_a_changed_order_of_memory(native, dtype, back, monkeypatch):
    """Steps, channels_last, steps (and back): the bits of a parameter that never changed, also in the state."""
    both_paths(monkeypatch, native)
    stay, move = image_kernel(dtype=dtype), image_kernel(dtype=dtype)
    other = [image_kernel(1, (5, 7), dtype) for _ in range(2)]
    a, b = (optim.AdamW([o, p], lr=LR) for p, o in ((stay, other[0]), (move, other[1])))
    for t in range(6):
        if t == 2:
            move.data = move.data.to(memory_format=LAST)
        if t == 4 and back:
            move.data = move.data.contiguous()
        take(a, [stay, other[0]], t)
        take(b, [move, other[1]], t)
        assert torch.equal(stay.detach(), move.detach()) and torch.equal(*(o.detach() for o in other))
        for name in ("exp_avg", "exp_avg_sq"):
            mine = b.state[move][name]
            assert torch.equal(a.state[stay][name], mine) and mine.stride() == move.stride()
            assert mine.data_ptr() == b._buffers[0][name][64:].data_ptr()


@pytest.mark.parametrize("native", [True, False])
def test_8_bit_moments_refuse_a_changed_order_of_memory(native, monkeypatch):
    """A block's elements share a power, so codes cannot be moved; before the first step they are all zero."""
    both_paths(monkeypatch, native)
    p, q = image_kernel(), image_kernel(1)
    opt = optim.AdamW([q, p], lr=LR, state_bits=8)
    p.data = p.data.to(memory_format=LAST)
    take(opt, [q, p], 0)
    take(opt, [q, p], 1)
    kept = [t.detach().clone() for t in (p, q)]
    p.data = p.data.contiguous()
    for t in (p, q):
        t.grad = torch.ones_like(t)
    with pytest.raises(ValueError, match="order"):
        opt.step()
    assert torch.equal(p.detach(), kept[0]) and torch.equal(q.detach(), kept[1])
    assert [int(opt.state[t]["step"]) for t in (p, q)] == [2, 2]
    p.data = p.data.to(memory_format=LAST)
    opt.step()
    assert not torch.equal(p.detach(), kept[0])


@pytest.mark.parametrize("native", [True, False])
@pytest.mark.parametrize("bits", [8, 32])
def test_channels_last_parameters_over_several_steps(native, bits, monkeypatch):
    """As the same elements in a dense parameter of that order of memory, whatever the order the gradient comes in."""
    both_paths(monkeypatch, native)
    last = image_kernel()
    dense = torch.nn.Parameter(last.detach().permute(0, 2, 3, 1).contiguous())
    last.data = last.data.to(memory_format=LAST)
    a, b = (optim.AdamW([p], lr=LR, state_bits=bits, seed=4) for p in (last, dense))
    for t in range(4):
        last.grad = some_grad(last, t)  # in the order of its shape
        dense.grad = last.grad.permute(0, 2, 3, 1).contiguous()
        a.step()
        b.step()
        assert torch.equal(last.detach().permute(0, 2, 3, 1), dense.detach())


def test_a_reshaped_parameter_and_one_sided_dimensions_keep_their_order():
    """The order of memory alone counts: a flattened dense parameter, or other strides of a dimension of 1."""
    p, q = image_kernel(), image_kernel()
    a, b = (optim.AdamW([t], lr=LR, state_bits=8) for t in (p, q))
    take(a, [p], 0)
    take(b, [q], 0)
    q.grad = None
    q.data = q.data.view(-1)
    p.grad = some_grad(p, 1)
    q.grad = some_grad(p, 1).view(-1)
    a.step()
    b.step()
    assert torch.equal(p.detach().view(-1), q.detach())
    r = torch.nn.Parameter(torch.randn(4, 1, 5, 5, device=DEV))
    opt = optim.AdamW([r], lr=LR, state_bits=8)
    take(opt, [r], 0)
    r.data = r.data.to(memory_format=LAST)
    take(opt, [r], 1)
    assert int(opt.state[r]["step"]) == 2


@pytest.mark.parametrize("native", [True, False])
@pytest.mark.parametrize("bits", [8, 32])
def test_parameters_in_any_dense_order(native, bits, monkeypatch):
    """A transposed matrix fills its memory too."""
    both_paths(monkeypatch, native)
    base = torch.randn(70, 33, device=DEV)
    turned, plain = torch.nn.Parameter(base.clone().t()), torch.nn.Parameter(base.clone())
    cube = torch.nn.Parameter(torch.randn(5, 6, 7, device=DEV).permute(2, 0, 1))
    a, b = optim.AdamW([turned, cube], lr=LR, state_bits=bits), optim.AdamW([plain], lr=LR, state_bits=bits)
    assert not turned.is_contiguous() and not cube.is_contiguous()
    for t in range(3):
        plain.grad = some_grad(plain, t)
        turned.grad = plain.grad.t().contiguous()  # brought into the parameter's order
        cube.grad = some_grad(cube, t)
        before = cube.detach().double().cpu()
        a.step()
        b.step()
        assert torch.equal(turned.detach().t(), plain.detach())
        if t == 0:
            zero = torch.zeros(cube.shape, dtype=torch.float64)
            ref.close(cube, ref.adamw(before, cube.grad.double().cpu(), zero, zero, 1, LR, (0.9, 0.999), 1e-8, 1e-2)[0], "f32", 8)


# ----------------------------------------------------------------------------
# saved states
# ----------------------------------------------------------------------------

@pytest.mark.parametrize("first,then", [("dense", "last"), ("last", "dense"), ("last", "last")])
def test_8_bit_states_of_another_order_of_memory_are_refused(first, then):
    make = lambda order: torch.nn.Parameter(  # noqa: E731
        image_kernel().detach().contiguous(memory_format=LAST if order == "last" else torch.contiguous_format))
    p, q = make(first), make(then)
    a, b = (optim.AdamW([t], lr=LR, state_bits=8, seed=3) for t in (p, q))
    take(a, [p], 0)
    saved = copy.deepcopy(a.state_dict())
    if first != then:
        with pytest.raises(ValueError, match="order"):
            b.load_state_dict(saved)
        assert int(b.state[q]["step"]) == 0
        return
    q.data.copy_(p.data)
    b.load_state_dict(saved)
    take(a, [p], 1)
    take(b, [q], 1)
    assert torch.equal(p.detach(), q.detach())


def test_32_bit_states_go_between_orders_of_memory():
    p, q = image_kernel(), image_kernel()
    q.data = q.data.to(memory_format=LAST)
    a, b = (optim.AdamW([t], lr=LR) for t in (p, q))
    take(a, [p], 0)
    q.data.copy_(p.data)
    b.load_state_dict(copy.deepcopy(a.state_dict()))
    take(a, [p], 1)
    take(b, [q], 1)
    assert torch.equal(p.detach(), q.detach())
    assert torch.equal(a.state[p]["exp_avg"], b.state[q]["exp_avg"])


def test_states_from_before_the_order_was_kept():
    """They have no "order": dense parameters'."""
    p = image_kernel()
    opt = optim.AdamW([p], lr=LR, state_bits=8)
    take(opt, [p], 0)
    saved = copy.deepcopy(opt.state_dict())
    for state in saved["state"].values():
        state.pop("order", None)
    saved.pop("seed", None)
    q = torch.nn.Parameter(p.detach().clone())
    other = optim.AdamW([q], lr=LR, state_bits=8)
    other.load_state_dict(saved)
    take(opt, [p], 1)
    take(other, [q], 1)
    assert torch.equal(p.detach(), q.detach())
    r = torch.nn.Parameter(p.detach().to(memory_format=LAST))
    with pytest.raises(ValueError, match="order"):
        optim.AdamW([r], lr=LR, state_bits=8).load_state_dict(saved)
