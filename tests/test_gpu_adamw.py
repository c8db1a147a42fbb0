"""AdamW on the GPU against float64 steps of the same stored values."""
import copy

import pytest
import torch

from paper_2608_10805_amd import binding, optim

from tests import _block as ref

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
LR, BETAS, EPS = 1e-2, (0.9, 0.999), 1e-8
# one element, around the block of 64, around a workgroup's share, kernels, a larger matrix
SHAPES = [(1,), (), (63,), (64,), (65,), (3, 5, 5), (2047,), (2048,), (8191,), (8193,), (127, 129), (300, 301)]


def make(shapes, dtype="f32", seed=0, grad_scale=1e-2):
    g = torch.Generator(device=DEV).manual_seed(seed)
    ps = [torch.nn.Parameter((torch.randn(s, generator=g, device=DEV)).to(ref.DTYPES[dtype])) for s in shapes]
    for p in ps:
        p.grad = (torch.randn(p.shape, generator=g, device=DEV) * grad_scale).to(p.dtype)
    return ps


def d(t):
    return t.detach().double().cpu()


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("scale", [None, 0.37])
def test_steps_with_32_bit_moments(dtype, scale):
    ps = make(SHAPES, dtype)
    opt = optim.AdamW([{"params": ps[::2]}, {"params": ps[1::2], "weight_decay": 0.0, "lr": 3e-3}], lr=LR, betas=BETAS,
                      eps=EPS, weight_decay=0.1)
    gs = torch.tensor([scale], device=DEV) if scale is not None else None
    m = [torch.zeros(p.shape, dtype=torch.float64) for p in ps]
    v = [torch.zeros(p.shape, dtype=torch.float64) for p in ps]
    for t in range(1, 4):
        before = [d(p) for p in ps]
        opt.step(grad_scale=gs)
        for i, p in enumerate(ps):
            lr, decay = (LR, 0.1) if i % 2 == 0 else (3e-3, 0.0)
            # every step from the stored parameter and the float32 moments, so that roundings do not add up
            want, m[i], v[i] = ref.adamw(before[i], d(p.grad) * (float(gs) if scale else 1.0), m[i], v[i], t, lr, BETAS, EPS, decay)
            # the parameter: its own product and sum, and the update (at most 10 lr) to 16 roundings
            ref.close(p, want, dtype, 4, scale=float(want.abs().max()) + 40 * lr if want.numel() else None)
            for name, exact in (("exp_avg", m[i]), ("exp_avg_sq", v[i])):
                # in units of its own largest value, a few roundings a step
                ref.close(opt.state[p][name], exact, "f32", 8 * t)
                assert opt.state[p][name].shape == p.shape
            assert int(opt.state[p]["step"]) == t
        for p in ps:
            p.grad = p.grad.flip(0) if p.dim() else -p.grad


def test_many_tensors_and_groups_reach_every_element():
    """More tensors and more groups than one launch takes."""
    shapes = [(7 + i % 90,) for i in range(400)]
    ps = make(shapes)
    before = [d(p) for p in ps]
    groups = [{"params": ps[i::20], "lr": 1e-3 * (i + 1)} for i in range(20)]
    opt = optim.AdamW(groups, betas=BETAS, eps=EPS, weight_decay=0.0)
    opt.step()
    zero = torch.zeros(1, dtype=torch.float64)
    for i, p in enumerate(ps):
        want, _, _ = ref.adamw(before[i], d(p.grad), zero, zero, 1, 1e-3 * (i % 20 + 1), BETAS, EPS, 0.0)
        ref.close(p, want, "f32", 8)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_steps_with_8_bit_moments(dtype):
    """Each step against a float64 step from the same codes: the parameter as with exact moments, each moment one of
    the two codes around its exact value, and which one as the given random bits say."""
    ps = make(SHAPES, dtype)
    opt = optim.AdamW(ps, lr=LR, betas=BETAS, eps=EPS, weight_decay=0.1, state_bits=8, seed=5)
    buffers = opt._buffers[0]
    for t in range(1, 5):
        before = [d(p) for p in ps]
        old = [(ref.decode(buffers["exp_avg"], buffers["exp_avg_scale"], True),
                ref.decode(buffers["exp_avg_sq"], buffers["exp_avg_sq_scale"], False))][0]
        opt.step()
        new = (ref.decode(buffers["exp_avg"], buffers["exp_avg_scale"], True),
               ref.decode(buffers["exp_avg_sq"], buffers["exp_avg_sq_scale"], False))
        shown = opt.moments()[0]
        for values, exact, bits in zip(shown, new, (4, 5)):
            assert values.dtype == torch.bfloat16 and torch.equal(d(values), exact)
        key = optim.rounding_key(5, t, 0)
        for i, p in enumerate(ps):
            n, at = p.numel(), buffers["offsets"][i]
            want, m, v = ref.adamw(before[i].reshape(-1), d(p.grad).reshape(-1), old[0][at:at + n], old[1][at:at + n], t,
                                   LR, BETAS, EPS, 0.1)
            ref.close(p.detach().reshape(-1), want, dtype, 4, scale=float(want.abs().max()) + 40 * LR)
            place = torch.arange(at, at + n)
            x = (place * 0x9E3779B1 + key) & 0xFFFFFFFF
            x = ((x ^ (x >> 15)) * 0x85EBCA6B) & 0xFFFFFFFF
            x = ((x ^ (x >> 13)) * 0xC2B2AE35) & 0xFFFFFFFF
            x = x ^ (x >> 16)
            for got, exact, bits, r in ((new[0], m, 4, x & 0xFFFF), (new[1], v, 5, x >> 16)):
                got, top = got[at:at + n], 2 ** bits - 2
                pad = torch.cat([exact, torch.zeros(-n % 64, dtype=torch.float64)]).view(-1, 64)
                largest = (torch.frexp(pad.abs().amax(1))[1] - 1).repeat_interleave(64)[:n].double()
                step = 2.0 ** (torch.maximum((torch.frexp(exact)[1] - 1).double(), largest - top + 1) - 3)
                down = (exact.abs() / step).floor() * step
                rest = (exact.abs() - down) / step + (r.double() + 0.5) / 65536
                # float32 places the value between the codes to 2^-20 of a step: within that of 1 either may come
                sure = (rest - 1).abs() > 2.0 ** -18
                expected = torch.where(rest >= 1, down + step, down) * exact.sign()
                assert bool(((got - exact).abs() <= step * (1 + 2.0 ** -18)).all())
                assert torch.equal(got[sure], expected[sure])
                assert bool(sure.double().mean() > 0.99) or n < 1000
            assert int(opt.state[p]["step"]) == t
        assert bool((buffers["exp_avg"][buffers["offsets"][1] + 1:buffers["offsets"][2]] == 0).all())  # the rest of a block


def test_8_bit_moments_are_unbiased():
    """With beta2 = 0.999 a step moves v by less than half of a code's distance: rounding to nearest would hold it.
    Rounded at random, the mean over many elements follows the exact recursion: 65536 elements whose codes are at most
    1/8 apart average to within 1/8 / 256 * 8 per sqrt(step)."""
    n, steps = 65536, 300
    p = torch.nn.Parameter(torch.zeros(n, device=DEV))
    opt = optim.AdamW([p], lr=0.0, betas=BETAS, eps=EPS, weight_decay=0.0, state_bits=8)
    v = m = 0.0
    for t in range(steps):
        g = 1.0 if t < 50 else 0.5
        p.grad = torch.full((n,), g, device=DEV)
        opt.step()
        m, v = BETAS[0] * m + (1 - BETAS[0]) * g, BETAS[1] * v + (1 - BETAS[1]) * g * g
    got_m, got_v = (float(t.double().mean()) for t in opt.moments(torch.float32)[0])
    assert abs(got_m - m) < 0.01 * m and abs(got_v - v) < 0.02 * v


def test_8_bit_moments_of_a_wide_range():
    """A block of magnitudes over twelve decades: each code is within 1/8 of its value, or within one step of the
    smallest, 2^-16 of the largest for m and 2^-32 for v."""
    p = torch.nn.Parameter(torch.zeros(64, device=DEV))
    p.grad = 10.0 ** torch.linspace(-9, 3, 64, device=DEV)
    opt = optim.AdamW([p], lr=1e-3, betas=(0.0, 0.0), state_bits=8)
    opt.step()
    m, v = (d(t) for t in opt.moments(torch.float32)[0])
    g = d(p.grad)
    assert bool(((m - g).abs() <= g / 8 + 1024 * 2.0 ** -16).all())
    assert bool(((v - g * g).abs() <= g * g / 8 + 2.0 ** 20 * 2.0 ** -32).all())


@pytest.mark.parametrize("bits", [8, 32])
@pytest.mark.parametrize("bad", [float("inf"), float("nan")])
def test_non_finite_gradients(bits, bad):
    """They spoil their element (8 bits: the block of 64 it lies in, from the next step on) and nothing else."""
    ps = make([(200,)])
    good = make([(200,)])
    a, b = (optim.AdamW(x, lr=LR, state_bits=bits) for x in (ps, good))
    ps[0].grad[70] = bad
    a.step()
    b.step()
    other = torch.arange(200) != 70
    assert bool(ps[0][70].isnan()) and torch.equal(ps[0].detach()[other], good[0].detach()[other])
    ps[0].grad.copy_(good[0].grad)
    a.step()
    b.step()
    if bits == 8:
        other = (torch.arange(200) < 64) | (torch.arange(200) >= 128)
        assert bool(ps[0].detach()[64:128].isnan().all())
    assert torch.equal(ps[0].detach()[other], good[0].detach()[other])


@pytest.mark.parametrize("bits", [8, 32])
@pytest.mark.parametrize("eps", [0.0, 2.0 ** -80])
def test_second_moments_below_the_normal_numbers(bits, eps):
    """Gradients whose squares are subnormal, with an eps that does not hide them. Every moment is a power of two,
    which float32 holds exactly."""
    for power in (-55, -60, -64, -68):  # v = 2^-120, 2^-130, 2^-138, 2^-146
        p = torch.nn.Parameter(torch.ones(200, device=DEV))
        p.grad = torch.full((200,), 2.0 ** power, device=DEV)
        optim.AdamW([p], lr=0.125, betas=(0.5, 1 - 2.0 ** -10), eps=eps, weight_decay=0.0, state_bits=bits).step()
        zero = torch.zeros(1, dtype=torch.float64)
        want, _, _ = ref.adamw(torch.ones(200, dtype=torch.float64), d(p.grad), zero, zero, 1, 0.125,
                               (0.5, 1 - 2.0 ** -10), eps, 0.0)
        ref.close(p, want, "f32", 8)


def test_zero_gradients_and_a_zero_eps():
    p = torch.nn.Parameter(torch.ones(100, device=DEV))
    p.grad = torch.zeros(100, device=DEV)
    for bits in (8, 32):
        opt = optim.AdamW([p], lr=0.1, weight_decay=0.0, state_bits=bits)
        opt.step()
        assert torch.equal(p.detach(), torch.ones(100, device=DEV))
    optim.AdamW([p], lr=0.1, eps=0.0).step()
    assert bool(p.isnan().all())  # 0 / 0, as the formula has it


@pytest.mark.parametrize("bits", [8, 32])
def test_the_same_step_gives_the_same_bits(bits):
    runs = []
    for _ in range(2):
        ps = make(SHAPES, seed=9)
        opt = optim.AdamW(ps, lr=LR, state_bits=bits, seed=3)
        for _ in range(3):
            opt.step()
        runs.append([p.detach().clone() for p in ps] + [t for pair in opt.moments() for t in pair])
    assert all(torch.equal(a, b) for a, b in zip(*runs))


@pytest.mark.parametrize("bits", [8, 32])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_unaligned_and_channels_last_parameters(bits, dtype):
    """Parameters and gradients that begin off a vector's alignment, or lie in another order, step as dense ones do."""
    base = make([(1, 301), (8, 6, 3, 3)], dtype)
    dense = [torch.nn.Parameter(p.detach().clone()) for p in base]
    for p, q in zip(dense, base):
        p.grad = q.grad.clone()
    room = torch.zeros(600, dtype=base[0].dtype, device=DEV)
    odd = torch.nn.Parameter(room[1:302].view(1, 301).copy_(base[0].detach()))
    odd.grad = torch.zeros(400, dtype=odd.dtype, device=DEV)[3:304].view(1, 301).copy_(base[0].grad)
    last = torch.nn.Parameter(base[1].detach().contiguous(memory_format=torch.channels_last))
    last.grad = base[1].grad.clone()  # in the dense order: brought into the parameter's
    a, b = optim.AdamW(dense, lr=LR, state_bits=32), optim.AdamW([odd, last], lr=LR, state_bits=32)
    a.step()
    b.step()
    assert all(torch.equal(x.detach(), y.detach()) for x, y in zip(dense, (odd, last)))
    assert float(room[0].abs() + room[302:].abs().sum()) == 0
    if bits == 8:
        a, b = optim.AdamW(dense, lr=LR, state_bits=8), optim.AdamW([odd, last], lr=LR, state_bits=8)
        a.step()
        b.step()
        assert torch.equal(dense[0].detach(), odd.detach())
        # the first step's update does not depend on the codes
        assert torch.equal(dense[1].detach(), last.detach())


@pytest.mark.parametrize("bits", [8, 32])
def test_the_native_host_path_is_the_python_one(bits, monkeypatch):
    """The same library calls, so the same bits, whichever path takes the step."""
    from paper_2608_10805_amd import autograd

    runs = []
    for native in (True, False):
        ps = make(SHAPES) + make(SHAPES[3:7], "bf16", seed=1)
        ps[4].grad = None
        opt = optim.AdamW([{"params": ps[:5]}, {"params": ps[5:], "lr": 0.3}], lr=LR, state_bits=bits, seed=8)
        assert autograd._block and all(opt._native)
        if native:
            monkeypatch.setattr(opt, "_step", lambda scale: pytest.fail("left to Python"))
        else:
            opt._native = [None] * 2
            if bits == 8:
                with pytest.raises(ValueError, match="float32, bfloat16"):
                    opt.moments(torch.float64)
        for _ in range(2):
            opt.step(grad_scale=torch.tensor(0.5, device=DEV))
        runs.append([p.detach().clone() for p in ps] + [t for pair in opt.moments() for t in pair] +
                    [opt.state[p]["step"].clone() for p in ps])
    assert all(torch.equal(a, b) for a, b in zip(*runs))


def test_parameters_without_gradients_are_left_alone():
    ps = make([(100,), (100,), (100,)])
    ps[1].grad = None
    kept = ps[1].detach().clone()
    opt = optim.AdamW(ps, lr=LR, weight_decay=0.1)
    opt.step()
    assert torch.equal(ps[1].detach(), kept) and [int(opt.state[p]["step"]) for p in ps] == [1, 0, 1]
    ps[1].grad = torch.ones(100, device=DEV)
    before = [d(p) for p in ps]
    m = [d(opt.state[p]["exp_avg"]) for p in ps]
    v = [d(opt.state[p]["exp_avg_sq"]) for p in ps]
    opt.step()  # two steps and one step of the same group
    for i, (p, t) in enumerate(zip(ps, (2, 1, 2))):
        ref.close(p, ref.adamw(before[i], d(p.grad), m[i], v[i], t, LR, BETAS, EPS, 0.1)[0], "f32", 8)
    for p in ps:
        p.grad = None
    kept = [p.detach().clone() for p in ps]
    opt.step()
    assert all(torch.equal(p.detach(), k) for p, k in zip(ps, kept))


@pytest.mark.parametrize("bits", [8, 32])
def test_state_dict_round_trip(bits):
    ps = make([(100,), (3, 70)])
    opt = optim.AdamW([{"params": ps[:1]}, {"params": ps[1:], "lr": 0.5}], lr=LR, state_bits=bits, seed=2)
    opt.step()
    saved, kept = copy.deepcopy(opt.state_dict()), [p.detach().clone() for p in ps]
    opt.step()
    want = [p.detach().clone() for p in ps]
    for p, k in zip(ps, kept):
        p.data.copy_(k)
    other = optim.AdamW([{"params": ps[:1]}, {"params": ps[1:]}], lr=0.9, state_bits=bits, seed=2)
    other.load_state_dict(saved)
    assert other.param_groups[1]["lr"] == 0.5
    other.step()
    assert all(torch.equal(p.detach(), w) for p, w in zip(ps, want))
    with pytest.raises(ValueError, match="other bits|not of these"):
        optim.AdamW([{"params": ps[:1]}, {"params": ps[1:]}], state_bits=40 - bits).load_state_dict(saved)
    with pytest.raises(ValueError, match="other parameter groups"):
        optim.AdamW(ps, state_bits=bits).load_state_dict(saved)


def test_a_scheduler_a_closure_and_mixed_types():
    ps = make([(10,)]) + make([(20,)], "bf16") + make([(30,)], "f16")
    opt = optim.AdamW(ps, lr=1.0, weight_decay=0.0)
    sched = torch.optim.lr_scheduler.LambdaLR(opt, lambda t: 0.5 ** t)
    before = [d(p) for p in ps]
    assert opt.step(lambda: 42) == 42
    for p, b in zip(ps, before):  # the first update has the size lr
        assert bool(((d(p) - b).abs() - 1.0).abs().max() < 0.02)
    sched.step()
    assert opt.param_groups[0]["lr"] == 0.5


def test_a_step_is_seen_by_autograd_and_refused_in_a_capture():
    p = torch.nn.Parameter(torch.ones(8, device=DEV))
    y = (p * p).sum()
    p.grad = torch.ones(8, device=DEV)
    opt = optim.AdamW([p])
    opt.step()
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.backward()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        z = p * 2
        with pytest.raises(RuntimeError, match="captured"):
            opt.step()
    assert int(opt.state[p]["step"]) == 1 and z.shape == p.shape


@pytest.mark.parametrize("mutate,match", [
    (lambda p: setattr(p, "grad", torch.ones(4, 4, device=DEV).to_sparse()), "dense"),
    (lambda p: setattr(p, "data", torch.ones(5, 5, device=DEV)), "changed"),
])
def test_step_refusals(mutate, match):
    p, q = (torch.nn.Parameter(torch.ones(4, 4, device=DEV)) for _ in range(2))
    opt = optim.AdamW([q, p])
    q.grad = torch.ones(4, 4, device=DEV)
    mutate(p)
    if p.grad is None:
        p.grad = torch.ones(p.shape, device=DEV)
    with pytest.raises((ValueError, RuntimeError), match=match):
        opt.step()
    assert torch.equal(q.detach(), torch.ones(4, 4, device=DEV)) and int(opt.state[q]["step"]) == 0


@pytest.mark.parametrize("kwargs,match", [
    (dict(lr=-1.0), "lr"), (dict(eps=-1e-8), "eps"), (dict(weight_decay=-1.0), "weight_decay"),
    (dict(betas=(1.0, 0.9)), "betas"), (dict(betas=(0.9, -0.1)), "betas"), (dict(state_bits=16), "state_bits"),
    (dict(lr=float("nan")), "lr"),
])
def test_constructor_refusals(kwargs, match):
    with pytest.raises(ValueError, match=match):
        optim.AdamW([torch.nn.Parameter(torch.ones(4, device=DEV))], **kwargs)


def test_parameter_refusals():
    for p, match in ((torch.ones(4), "GPU"), (torch.ones(4, dtype=torch.float64, device=DEV), "float32, bfloat16"),
                     (torch.ones(4, 8, device=DEV)[:, ::2], "fill")):
        with pytest.raises(ValueError, match=match):
            optim.AdamW([torch.nn.Parameter(p)])
    good = torch.nn.Parameter(torch.ones(4, device=DEV))
    opt = optim.AdamW([good])
    with pytest.raises(ValueError, match="GPU"):
        opt.add_param_group({"params": [torch.nn.Parameter(torch.ones(4))]})
    good.grad = torch.ones(4, device=DEV)
    opt.step()
    for bad in (torch.ones(2, device=DEV), torch.ones(1, dtype=torch.float64, device=DEV), torch.ones(1)):
        with pytest.raises(ValueError, match="grad_scale"):
            opt.step(grad_scale=bad)
    assert int(opt.state[good]["step"]) == 1 and len(opt.param_groups) == 1


def test_moments_beyond_32_bits_of_elements():
    """Codes from the 2^32nd on: the last block is where the offsets are largest."""
    n = (1 << 32) + 128
    m, v = torch.zeros(n, dtype=torch.uint8, device=DEV), torch.zeros(n, dtype=torch.uint8, device=DEV)
    ms = torch.full((n // 64,), 127, dtype=torch.uint8, device=DEV)
    p, g = torch.ones(128, device=DEV), torch.full((128,), 2.0, device=DEV)
    group = binding.AdamWGroup(0.1, 0.5, 0.5, 0.0, 0.0, 1, 7, m.data_ptr(), v.data_ptr(), ms.data_ptr(), ms.data_ptr())
    other = torch.full_like(ms, 127)
    group.exp_avg_sq_scale = other.data_ptr()
    tensor = binding.AdamWTensor(p.data_ptr(), g.data_ptr(), 128, 1 << 32, 0)
    assert binding.wtconv_adamw_step([group], [tensor], 0, 8, None, torch.cuda.current_stream().cuda_stream) == 0
    tail = slice((1 << 32), n)
    assert torch.equal(ref.decode(m[tail], ms[-2:], True), torch.full((128,), 1.0, dtype=torch.float64))
    assert torch.equal(ref.decode(v[tail], other[-2:], False), torch.full((128,), 2.0, dtype=torch.float64))
    ref.close(p, torch.full((128,), 0.9, dtype=torch.float64), "f32", 4)
    assert int(m[:1 << 20].sum()) == 0
