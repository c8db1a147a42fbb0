"""Layer norm and scaled residual on the GPU against float64 references of the
same stored values, at the sizes, layouts and values where they can go wrong."""
import pytest
import torch

from paper_2608_10805_amd import autograd, binding

from tests import _block as ref

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
LAYOUTS = {"rows": (-1, -1), "turned": (1, -1), "planes": (1, 1)}


def gen(seed=0):
    return torch.Generator(device=DEV).manual_seed(seed)


def normal(g, shape, dtype="f32", scale=1.0, shift=0.0):
    return (torch.randn(shape, generator=g, device=DEV) * scale + shift).to(ref.DTYPES[dtype])


def norm_problem(layout, B, C, S, dtype, affine=True, seed=0):
    g = gen(seed)
    cin, cout = LAYOUTS[layout]
    sp = S if isinstance(S, tuple) else (S,)
    shape, rows = (B, C, *sp), (B, *sp, C)
    x = normal(g, rows if cin == -1 else shape, dtype, 1.5, 0.3)
    dy = normal(g, rows if cout == -1 else shape, dtype)
    w = normal(g, (C,), scale=0.5, shift=1.0) if affine else None
    b = normal(g, (C,), scale=0.5) if affine else None
    return x, dy, w, b


def reference(x, dy, w, b, layout, eps):
    cin, cout = LAYOUTS[layout]
    d = lambda t: t.detach().double().cpu() if t is not None else None  # noqa: E731
    y, xhat, rstd = ref.norm(ref.to_rows(x, cin), d(w), d(b), eps)
    dx, dw, db = ref.norm_grads(ref.to_rows(dy, cout), xhat, rstd, d(w))
    return ref.from_rows(y, dy.shape, cout), ref.from_rows(dx, x.shape, cin), dw, db, rstd


def check_norm(x, dy, w, b, layout, dtype, eps=1e-6):
    cin, cout = LAYOUTS[layout]
    leaves = [t for t in (x, w, b) if t is not None]
    for t in leaves:
        t.requires_grad_(True)
    y = autograd.layer_norm(x, w, b, eps, cin, cout)
    got = torch.autograd.grad(y, leaves, dy)
    want_y, want_dx, want_dw, want_db, rstd = reference(x, dy, w, b, layout, eps)
    assert y.dtype == x.dtype and y.shape == dy.shape
    C = x.shape[cin]
    # terms of one pixel are C long, those of a weight's gradient as long as the pixels: in units of one rounding of
    # the largest value, the row sums (spread over lanes) stay below 64 + C / 16 roundings
    row = 64 + C / 16
    ref.close(y, want_y, dtype, row)
    ref.close(got[0], want_dx, dtype, row, scale=float(dy.float().abs().max() * rstd.max() * (w.detach().abs().max() if w is not None else 1)))
    if w is not None:
        # sums over all pixels of products near 1: a rounding of each term's size and of the running sum's
        n = max(1, x.numel() // C)
        ref.close(got[1], want_dw, "f32", 64, scale=float(n) ** 0.5 * 8 + float(want_dw.abs().max()))
        ref.close(got[2], want_db, "f32", 64, scale=float(n) ** 0.5 * 8 + float(want_db.abs().max()))


@pytest.mark.parametrize("layout", list(LAYOUTS))
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("B,C,S", [(1, 1, 1), (1, 2, 3), (2, 3, 49), (3, 8, 64), (2, 31, (5, 13)), (1, 96, 196),
                                   (5, 96, (7, 7)), (2, 127, (9, 11)), (1, 129, 65), (2, 192, (14, 14)), (3, 256, 16),
                                   (2, 384, (7, 9)), (2, 768, 49), (1, 1000, 33), (1, 1025, 20), (1, 2048, 12)])
def test_norm(layout, dtype, B, C, S):
    check_norm(*norm_problem(layout, B, C, S, dtype), layout, dtype)


@pytest.mark.parametrize("layout", list(LAYOUTS))
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,C,S", [(1, 5000, 9), (1, 20001, 3), (1, 4099, 70)])
def test_norm_of_many_channels(layout, dtype, B, C, S):
    check_norm(*norm_problem(layout, B, C, S, dtype), layout, dtype)


@pytest.mark.parametrize("layout", list(LAYOUTS))
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("B,C,S", [(32, 96, (28, 28)), (9, 33, (31, 45)), (64, 384, (7, 7)), (20, 64, (63, 95)),
                                   (7, 200, (16, 24))])
def test_norm_of_many_pixels(layout, dtype, B, C, S):
    check_norm(*norm_problem(layout, B, C, S, dtype, seed=3), layout, dtype)


@pytest.mark.parametrize("layout", list(LAYOUTS))
@pytest.mark.parametrize("C", [7, 96])
def test_norm_without_parameters(layout, C):
    x, dy, _, _ = norm_problem(layout, 2, C, 21, "f32", affine=False)
    check_norm(x, dy, None, None, layout, "f32")
    w = normal(gen(1), (C,), shift=1.0)
    for weight, bias in ((w, None), (None, w)):
        leaves = [x, w]
        for t in leaves:
            t.requires_grad_(True)
        y = autograd.layer_norm(x, weight, bias, 1e-5, *LAYOUTS[layout])
        got = torch.autograd.grad(y, leaves, dy)
        want = reference(x, dy, weight, bias, layout, 1e-5)
        ref.close(y, want[0], "f32", 64 + C / 16)
        ref.close(got[1], want[2] if weight is not None else want[3], "f32", 64, 8 * 42 ** 0.5)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("C", [24, 63, 96])
@pytest.mark.parametrize("shift", [0, 1])
def test_norm_of_strided_rows(dtype, C, shift):
    """Rows inside wider rows, from an element that is not aligned to vectors, for x and for dy."""
    wide = normal(gen(4), (3, 37, C + 5), dtype, 1.5)
    up = normal(gen(5), (3, 37, 2 * C + 3), dtype)
    x, dy = wide[..., shift:shift + C], up[..., shift:shift + C]
    w, b = normal(gen(6), (C,), shift=1.0), normal(gen(7), (C,))
    before = wide.clone()
    y, mean, rstd = binding.layer_norm_forward(x, w, b)
    dx, dw, db = binding.layer_norm_backward(dy, x, mean, rstd, w)
    want = reference(x, dy, w, b, "rows", 1e-6)
    ref.close(y, want[0], dtype, 70)
    ref.close(dx, want[1], dtype, 70, scale=float(dy.float().abs().max() * want[4].max() * w.abs().max()))
    ref.close(dw, want[2], "f32", 64, 8 * 111 ** 0.5 + float(want[2].abs().max()))
    ref.close(db, want[3], "f32", 64, 8 * 111 ** 0.5 + float(want[3].abs().max()))
    assert torch.equal(wide, before)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("B,C,S", [(3, 48, 64), (9, 96, 784), (40, 768, 196), (2, 128, 20)])
@pytest.mark.parametrize("more,shift", [(0, 0), (16, 8), (5, 0), (8, 1)])
def test_norm_of_planes_with_strided_gradient_rows(dtype, B, C, S, more, shift):
    """dy as rows inside wider rows, aligned to 16 bytes or not; all of the gradients, and each by itself."""
    x, dy, w, b = norm_problem("turned", B, C, S, dtype)
    pitch = C + more
    wide = torch.full((B * S * pitch + shift,), float("nan"), dtype=dy.dtype, device=DEV)[shift:].view(B, S, pitch)
    up = wide[..., :C]
    up.copy_(dy)
    _, mean, rstd = binding.layer_norm_forward(x, w, b, 1e-6, 1, -1)
    back = lambda t, **k: binding.layer_norm_backward(t, x, mean, rstd, w, 1e-6, 1, -1, **k)  # noqa: E731
    dx, dw, db = back(up)
    want = reference(x, dy, w, b, "turned", 1e-6)
    sums = 8 * float(B * S) ** 0.5
    ref.close(dx, want[1], dtype, 64 + C / 16, scale=float(dy.float().abs().max() * want[4].max() * w.abs().max()))
    ref.close(dw, want[2], "f32", 64, sums + float(want[2].abs().max()))
    ref.close(db, want[3], "f32", 64, sums + float(want[3].abs().max()))
    # neither the rows' place nor which gradients are asked for changes a result
    for a, o in zip(back(dy), (dx, dw, db)):
        assert torch.equal(a, o)
    assert torch.equal(back(up, need_dweight=False, need_dbias=False)[0], dx)
    assert all(torch.equal(a, o) for a, o in zip(back(up, need_dx=False)[1:], (dw, db)))


@pytest.mark.parametrize("layout", list(LAYOUTS))
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shift", [1, 2])
def test_norm_of_tensors_off_alignment(layout, dtype, shift):
    """Tensors that begin at an element that is not aligned to vectors."""
    x, dy, w, b = norm_problem(layout, 2, 48, (8, 8), dtype)
    move = lambda t: torch.cat([t.flatten()[:shift], t.flatten()])[shift:].view(t.shape)  # noqa: E731
    check_norm(move(x), move(dy), w, b, layout, dtype)


@pytest.mark.parametrize("layout", list(LAYOUTS))
def test_norm_of_nothing(layout):
    cin, cout = LAYOUTS[layout]
    x = torch.empty((0, 6, 5) if cin == 1 else (0, 5, 6), device=DEV, requires_grad=True)
    w = torch.ones(6, device=DEV, requires_grad=True)
    y = autograd.layer_norm(x, w, w, 1e-6, cin, cout)
    dx, dw = torch.autograd.grad(y, [x, w], torch.empty_like(y))
    assert y.numel() == 0 and dx.shape == x.shape and torch.equal(dw, torch.zeros_like(w))


@pytest.mark.parametrize("layout", list(LAYOUTS))
@pytest.mark.parametrize("C", [96, 100])
def test_norm_of_constant_and_of_shifted_pixels(layout, C):
    """A constant pixel has the variance 0 and the output `bias`; far from zero the mean's own rounding shows."""
    x, dy, w, b = norm_problem(layout, 2, C, 64, "f32")
    cin, cout = LAYOUTS[layout]
    y = autograd.layer_norm(torch.full_like(x, 3.25), w, b, 1e-6, cin, cout)
    assert torch.equal(ref.to_rows(y, cout), b.double().cpu().expand(128, C))
    shifted = x + 1000
    want = reference(shifted, dy, w, b, layout, 1e-6)
    # the mean, near 1000, is held to one float32 rounding and summed with at most 64
    ref.close(autograd.layer_norm(shifted, w, b, 1e-6, cin, cout), want[0], "f32", 64, 1000 * float(w.abs().max()))


@pytest.mark.parametrize("layout", list(LAYOUTS))
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("bad", [float("inf"), float("-inf"), float("nan")])
def test_norm_keeps_non_finite_values_to_their_pixel(layout, dtype, bad):
    cin, cout = LAYOUTS[layout]
    x, dy, w, b = norm_problem(layout, 2, 96, 100, dtype)
    clean = autograd.layer_norm(x, w, b, 1e-6, cin, cout)
    at = (1, 5, 17) if cin == 1 else (1, 17, 5)
    x[at] = bad
    y, mean, rstd = binding.layer_norm_forward(x, w, b, 1e-6, cin, cout)
    dx, dw, db = binding.layer_norm_backward(dy, x, mean, rstd, w, 1e-6, cin, cout)
    rows, other = ref.to_rows(y, cout), ref.to_rows(clean, cout)
    keep = torch.arange(200) != 117
    assert torch.equal(rows[keep], other[keep]) and bool(rows[117].isnan().all())
    drows = ref.to_rows(dx, cin)
    assert bool(drows[keep].isfinite().all()) and bool(drows[117].isnan().all())
    assert bool(dw.isnan().all()) and bool(db.isfinite().all())


@pytest.mark.parametrize("layout", list(LAYOUTS))
@pytest.mark.parametrize("B,C,S", [(8, 96, (28, 28)), (4, 384, (7, 7)), (2, 33, 65), (1, 5000, 9)])
def test_norm_gives_the_same_bits_again(layout, B, C, S):
    cin, cout = LAYOUTS[layout]
    x, dy, w, b = norm_problem(layout, B, C, S, "f32")
    out = []
    for _ in range(3):
        y, mean, rstd = binding.layer_norm_forward(x, w, b, 1e-6, cin, cout)
        out.append((y, mean, rstd, *binding.layer_norm_backward(dy, x, mean, rstd, w, 1e-6, cin, cout)))
    assert all(torch.equal(a, b) for other in out[1:] for a, b in zip(out[0], other))
    # each gradient alone, and the forward without statistics, are the same bits too
    y, mean, rstd = out[0][:3]
    assert torch.equal(binding.layer_norm_forward(x, w, b, 1e-6, cin, cout, stats=False)[0], y)
    for need in ((True, False, False), (False, True, False), (False, False, True)):
        got = binding.layer_norm_backward(dy, x, mean, rstd, w, 1e-6, cin, cout, *need)
        assert [t is not None for t in got] == list(need)
        assert all(torch.equal(a, b) for a, b in zip(got, out[0][3:]) if a is not None)


@pytest.mark.parametrize("layout", list(LAYOUTS))
def test_norm_gradient_against_differences(layout):
    """Central differences of the forward pass: with a step of 1/64 the formula's third-order error is below 1e-4 of
    the values, the rounding of sums of 60 outputs near 1 below 64 * 60 * 2^-24 / 2^-6."""
    cin, cout = LAYOUTS[layout]
    x, dy, w, b = norm_problem(layout, 1, 12, 5, "f32")
    leaves = [t.requires_grad_(True) for t in (x, w, b)]
    f = lambda: float((autograd.layer_norm(x, w, b, 0.1, cin, cout).double() * dy).sum())  # noqa: E731
    grads = torch.autograd.grad(autograd.layer_norm(x, w, b, 0.1, cin, cout), leaves, dy)
    h = 2.0 ** -6
    for t, g in zip(leaves, grads):
        flat = t.detach().view(-1)
        for i in range(0, flat.numel(), 7):
            old = flat[i].item()
            flat[i] = old + h
            up, hi = f(), flat[i].item()
            flat[i] = old - h
            down, lo = f(), flat[i].item()
            flat[i] = old
            assert abs((up - down) / (hi - lo) - g.view(-1)[i].item()) < 3e-2 * 2 ** -4 + 64 * 60 * 2.0 ** -24 / h


def test_norm_of_channels_last_planes_runs_as_rows():
    x, dy, w, b = norm_problem("planes", 2, 24, (6, 10), "f32")
    lay = x.contiguous(memory_format=torch.channels_last)
    y = autograd.layer_norm(lay, w, b, channel_dim=1)
    want = reference(x, dy, w, b, "planes", 1e-6)
    ref.close(y, want[0], "f32", 66)
    assert y.is_contiguous(memory_format=torch.channels_last)
    rows = autograd.layer_norm(lay, w, b, channel_dim=1, out_channel_dim=-1)
    assert rows.is_contiguous() and torch.equal(rows, y.movedim(1, -1))


def test_norm_of_an_expanded_gradient_and_of_transposed_rows():
    x, _, w, b = norm_problem("rows", 3, 20, 7, "f32")
    x.requires_grad_(True)
    autograd.layer_norm(x, w, b).sum().backward()  # the gradient of a sum has strides 0
    want = reference(x, torch.ones_like(x), w, b, "rows", 1e-6)
    ref.close(x.grad, want[1], "f32", 66, float(want[4].max()) * 3)
    t = x.detach().transpose(0, 1)
    assert torch.equal(autograd.layer_norm(t, w, b), autograd.layer_norm(x.detach(), w, b).transpose(0, 1))


def test_norm_on_another_stream():
    x, dy, w, b = norm_problem("turned", 8, 96, (28, 28), "f32")
    x.requires_grad_(True)
    want = autograd.layer_norm(x, w, b, channel_dim=1, out_channel_dim=-1)
    g = torch.autograd.grad(want, x, dy)[0]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        y = autograd.layer_norm(x, w, b, channel_dim=1, out_channel_dim=-1)
        h = torch.autograd.grad(y, x, dy)[0]
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(y, want) and torch.equal(g, h)


def test_norm_beyond_32_bits_of_elements():
    """More than 2^31 elements: the last rows and the last planes are where the offsets are largest."""
    C, n = 2048, (1 << 20) + 3
    x = torch.empty(n, C, dtype=torch.bfloat16, device=DEV).fill_(0.25)
    x[-3:] = normal(gen(8), (3, C), "bf16")
    y, _, _ = binding.layer_norm_forward(x)
    want = ref.norm(x[-3:].double().cpu(), None, None, 1e-6)[0]
    ref.close(y[-3:], want, "bf16", 200)
    planes = x.view(1, n, C)[:, :(1 << 20)].view(16, 1 << 16, C)  # [B, C = 65536, S = 2048]
    del y
    z, mean, rstd = binding.layer_norm_forward(planes, channel_dim=1)
    want = ref.norm(planes[-1, :, -2:].double().cpu().T, None, None, 1e-6)[0]
    ref.close(z[-1, :, -2:].T, want, "bf16", 64 + 65536 / 16)


@pytest.mark.parametrize("layout", ["turned", "planes"])
def test_norm_of_more_pixels_than_one_launch_takes(layout):
    """2^30 images of one pixel: 2^32 threads. Every pixel against the two values that a norm of two channels has."""
    n = (1 << 30) + 67
    x = torch.zeros(n, 2, 1, dtype=torch.float16, device=DEV)
    x[:, 0] = 1.0
    x[1::2, 0] = -3.0
    w, b = torch.tensor([1.0, 2.0], device=DEV), torch.tensor([0.5, -0.5], device=DEV)
    y, mean, rstd = binding.layer_norm_forward(x, w, b, 0.0, *LAYOUTS[layout])
    del x
    assert bool((mean[::2] == 0.5).all()) and bool((mean[1::2] == -1.5).all())
    for part, r in ((rstd[::2], 2.0), (rstd[1::2], 2 / 3)):  # to two roundings
        assert float((part - r).abs().max()) <= r * 2.0 ** -22
    del mean, rstd, part
    # xhat = 1 and -1, then -1 and 1; to two roundings of the result (at most 2.5)
    for part, want in ((y[::2], (1.5, -2.5)), (y[1::2], (-0.5, 1.5))):
        for c in (0, 1):
            v = part.reshape(part.shape[0], 2)[:, c]
            assert float(v.max()) - 2.0 ** -9 <= want[c] <= float(v.min()) + 2.0 ** -9
    torch.cuda.empty_cache()


def test_norm_of_more_rows_than_one_launch_takes():
    """2^30 rows of four lanes each: 2^32 threads. Rows of another kind lie at both ends and around the middle."""
    if torch.cuda.mem_get_info()[0] < 150e9:
        pytest.skip("needs 125 GB of GPU memory")
    n, C = (1 << 30) + 5, 25
    x = torch.zeros(n, C, dtype=torch.float16, device=DEV)
    places = [0, 1, n // 4, n // 2 - 1, n // 2, n // 2 + 1, 3 * (n // 4), n - 2, n - 1]
    some = normal(gen(12), (len(places), C), "f16")
    for p, row in zip(places, some):
        x[p].copy_(row)
    want = ref.norm(some.double().cpu(), None, None, 1e-6)
    y, mean, rstd = binding.layer_norm_forward(x, None, None, 1e-6)
    del x
    ref.close(torch.stack([y[p] for p in places]), want[0], "f16", 64)
    ref.close(torch.stack([rstd[p] for p in places]), want[2].view(-1), "f32", 64)
    assert int(mean.count_nonzero()) == len(places)
    others = torch.ones(n, dtype=torch.bool, device=DEV)
    others[places] = False
    for i in range(0, n, 1 << 26):
        part = y[i:i + (1 << 26)]
        assert not bool((part != 0).any(1).logical_and_(others[i:i + (1 << 26)]).any())
    del y, part
    torch.cuda.empty_cache()


def test_norm_in_a_graph():
    """A captured forward and backward, replayed with the program's own work between, gives the eager bits."""
    x, dy, w, b = norm_problem("turned", 4, 96, (14, 14), "f32")
    eager = lambda: (lambda y, m, r: (y, *binding.layer_norm_backward(  # noqa: E731
        dy, x, m, r, w, 1e-6, 1, -1)))(*binding.layer_norm_forward(x, w, b, 1e-6, 1, -1))
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        eager()
    torch.cuda.current_stream().wait_stream(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = eager()
    for i in range(4):
        x.copy_(normal(gen(20 + i), x.shape))
        want = eager()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(captured, want)), i


# ----------------------------------------------------------------------------
# scaled residual
# ----------------------------------------------------------------------------

def residual_problem(B, C, S, dtype, seed=0):
    g = gen(seed)
    sp = S if isinstance(S, tuple) else (S,)
    x, z = normal(g, (B, C, *sp), dtype), normal(g, (B, *sp, C), dtype)
    dy = normal(g, (B, C, *sp), dtype)
    gamma = normal(g, (C,), scale=0.5)
    keep = (torch.rand(B, generator=g, device=DEV) < 0.7).float() / 0.7
    return x, z, dy, gamma, keep


def check_residual(x, z, dy, gamma, keep, dtype):
    d = lambda t: t.detach().double().cpu() if t is not None else None  # noqa: E731
    leaves = [t.requires_grad_(True) for t in (x, z, gamma) if t is not None]
    y = autograd.scaled_residual(x, z, gamma, keep)
    got = torch.autograd.grad(y, leaves, dy)
    # three roundings: the factor, the product, the sum
    ref.close(y, ref.residual(d(x), d(z), d(gamma), d(keep)), dtype, 4, scale=32.0)
    dz, dgamma = ref.residual_grads(d(dy), d(z), d(gamma), d(keep))
    assert torch.equal(got[0], dy)
    ref.close(got[1], dz, dtype, 4)
    if gamma is not None:
        n = max(1, x.numel() // x.shape[1])
        ref.close(got[2], dgamma, "f32", 64, 8 * n ** 0.5 + float(dgamma.abs().max()))


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("B,C,S", [(1, 1, 1), (2, 1, 70), (1, 70, 1), (2, 3, 49), (3, 64, 64), (2, 65, (9, 7)),
                                   (1, 96, (56, 56)), (5, 127, (5, 13)), (4, 384, (7, 7)), (2, 770, 30),
                                   (16, 128, (28, 28)), (3, 40, (63, 95)), (1, 5000, 5)])
def test_residual(dtype, B, C, S):
    x, z, dy, gamma, keep = residual_problem(B, C, S, dtype)
    check_residual(x, z, dy, gamma, keep, dtype)
    check_residual(x, z, dy, gamma, None, dtype)
    check_residual(x, z, dy, None, keep, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shift", [1, 2])
def test_residual_of_tensors_off_alignment(dtype, shift):
    x, z, dy, gamma, keep = residual_problem(2, 48, (8, 8), dtype)
    move = lambda t: torch.cat([t.flatten()[:shift], t.flatten()])[shift:].view(t.shape)  # noqa: E731
    check_residual(move(x), move(z), move(dy), gamma, keep, dtype)


def test_residual_of_nothing():
    x = torch.empty(0, 6, 5, device=DEV, requires_grad=True)
    z, gamma = torch.empty(0, 5, 6, device=DEV), torch.ones(6, device=DEV, requires_grad=True)
    y = autograd.scaled_residual(x, z, gamma)
    dx, dg = torch.autograd.grad(y, [x, gamma], torch.empty_like(y))
    assert y.shape == x.shape and dx.shape == x.shape and torch.equal(dg, torch.zeros(6, device=DEV))


def test_residual_of_transposed_tensors_and_expanded_gradients():
    x, z, dy, gamma, keep = residual_problem(2, 12, (6, 10), "f32")
    want = autograd.scaled_residual(x, z, gamma, keep)
    assert torch.equal(want, autograd.scaled_residual(x.contiguous(memory_format=torch.channels_last),
                                                      z.transpose(1, 2).contiguous().transpose(1, 2), gamma, keep))
    z.requires_grad_(True)
    autograd.scaled_residual(x, z, gamma, keep).sum().backward()
    ref.close(z.grad, (keep.view(2, 1, 1, 1) * gamma).double().cpu().expand(z.shape), "f32", 2)


@pytest.mark.parametrize("bad", [float("inf"), float("nan")])
def test_residual_keeps_non_finite_values_to_their_element(bad):
    x, z, dy, gamma, _ = residual_problem(2, 70, 81, "f32")
    clean = autograd.scaled_residual(x, z, gamma)
    z[1, 3, 66] = bad
    y = autograd.scaled_residual(x, z, gamma)
    assert not bool(y[1, 66, 3].isfinite())
    y[1, 66, 3] = clean[1, 66, 3]
    assert torch.equal(y, clean)
    _, dg = binding.scaled_residual_backward(dy, z, gamma)
    assert not bool(dg[66].isfinite()) and int(dg.isfinite().sum()) == 69


def test_residual_gives_the_same_bits_again():
    x, z, dy, gamma, keep = residual_problem(16, 96, (28, 28), "f32")
    first = binding.scaled_residual_backward(dy, z, gamma, keep)
    for need in ((True, True), (True, False), (False, True)):
        again = binding.scaled_residual_backward(dy, z, gamma, keep, *need)
        assert all(torch.equal(a, b) for a, b in zip(again, first) if a is not None)
    assert torch.equal(binding.scaled_residual_backward(dy, None, gamma, keep, True, False)[0], first[0])


def test_residual_gradient_against_differences():
    """The residual is linear in z and in gamma: differences are exact up to the rounding of sums of values below 8."""
    x, z, dy, gamma, keep = residual_problem(2, 5, 6, "f32")
    dz, dg = binding.scaled_residual_backward(dy, z, gamma, keep)
    f = lambda: float((autograd.scaled_residual(x, z, gamma, keep).double() * dy).sum())  # noqa: E731
    for t, g in ((z, dz), (gamma, dg)):
        flat = t.view(-1)
        for i in range(0, flat.numel(), 4):
            old = flat[i].item()
            flat[i] = old + 0.5
            up, hi = f(), flat[i].item()
            flat[i] = old - 0.5
            down, lo = f(), flat[i].item()
            flat[i] = old
            assert abs((up - down) / (hi - lo) - g.view(-1)[i].item()) < 60 * 8 * 2.0 ** -22


# ----------------------------------------------------------------------------
# the native host path against the Python one: the same library calls, so the
# same bits, and the cases it leaves to Python
# ----------------------------------------------------------------------------

@pytest.mark.parametrize("layout", list(LAYOUTS))
@pytest.mark.parametrize("params", ["both", "weight", "bias", "none"])
@pytest.mark.parametrize("need_x", [True, False])
def test_native_norm_is_the_python_one(layout, params, need_x):
    x, dy, w, b = norm_problem(layout, 2, 24, (5, 7), "bf16")
    assert autograd.load_block(x), "the native host path is not built"
    x.requires_grad_(need_x)
    w = w.requires_grad_(True) if params in ("both", "weight") else None
    b = b.requires_grad_(True) if params in ("both", "bias") else None
    leaves = [t for t in (x, w, b) if t is not None and t.requires_grad]
    args = (x, w, b, 1e-6, *LAYOUTS[layout])
    assert autograd._block.layer_norm(*args) is not None
    fns = (autograd.layer_norm, autograd.LayerNormFunction.apply)
    got, want = ((y, *(torch.autograd.grad(y, leaves, dy) if leaves else ())) for y in (fn(*args) for fn in fns))
    assert len(got) == len(want) and all(torch.equal(a, b) for a, b in zip(got, want))
    with torch.no_grad():
        assert torch.equal(autograd.layer_norm(*args), want[0])
    if leaves:  # an upstream gradient in another order
        odd = dy.transpose(1, 2).contiguous().transpose(1, 2)
        assert torch.equal(torch.autograd.grad(autograd.layer_norm(*args), leaves[0], odd)[0], want[1])


@pytest.mark.parametrize("given", ["all", "gamma", "keep", "none"])
def test_native_residual_is_the_python_one(given):
    x, z, dy, gamma, keep = residual_problem(3, 20, (5, 7), "f16")
    gamma = gamma.requires_grad_(True) if given in ("all", "gamma") else None
    keep = keep if given in ("all", "keep") else None
    assert autograd._block.scaled_residual(x, z, gamma, keep) is not None
    for need in ((True, True), (False, True), (True, False), (False, False)):
        x.requires_grad_(need[0])
        z.requires_grad_(need[1])
        leaves = [t for t in (x, z, gamma) if t is not None and t.requires_grad]
        fns = (autograd.scaled_residual, autograd.ScaledResidualFunction.apply)
        got, want = ((y, *(torch.autograd.grad(y, leaves, dy) if leaves else ()))
                     for y in (fn(x, z, gamma, keep) for fn in fns))
        assert len(got) == len(want) and all(torch.equal(a, b) for a, b in zip(got, want))


class Tagged(torch.Tensor):
    """A subclass with torch functions of its own and no dispatch."""


def test_other_cases_take_the_python_path():
    from torch.utils._python_dispatch import TorchDispatchMode

    class Count(TorchDispatchMode):
        n = 0

        def __torch_dispatch__(self, func, types, args=(), kwargs=None):
            self.n += 1
            return func(*args, **(kwargs or {}))

    x, dy, w, b = norm_problem("turned", 2, 24, (5, 7), "f32")
    rows = x.movedim(1, -1).contiguous()
    ext = autograd._block
    for t in (x.transpose(2, 3), x.double(), x[:0], x.as_subclass(Tagged), x.cpu()):
        assert ext.layer_norm(t, w, b, 1e-6, 1, -1) is None
        assert ext.scaled_residual(t, rows, w, None) is None
    assert ext.layer_norm(x, w.half(), b, 1e-6, 1, -1) is None and ext.layer_norm(x, w, b, 1, 1, -1) is None
    assert ext.layer_norm(x, w, b[1:], 1e-6, 1, -1) is None and ext.layer_norm(x, w, b, 1e-6, 0, -1) is None
    assert ext.scaled_residual(x, rows[:1], w, None) is None and ext.scaled_residual(x, rows.half(), w, None) is None
    want = autograd.layer_norm(x, w, b, 1e-6, 1, -1)
    tagged = autograd.layer_norm(x.as_subclass(Tagged), w, b, 1e-6, 1, -1)
    assert type(tagged) is Tagged and torch.equal(tagged.as_subclass(torch.Tensor), want)
    with Count() as mode:
        assert torch.equal(autograd.layer_norm(x, w, b, 1e-6, 1, -1), want)
        assert torch.equal(autograd.scaled_residual(x, rows, w), autograd.ScaledResidualFunction.apply(x, rows, w, None))
    assert mode.n > 0
    for fn in (lambda v: autograd.layer_norm(v, w, b, 1e-6, 1, -1), lambda v: autograd.scaled_residual(v, rows, w)):
        with pytest.raises(Exception):  # forward-mode is refused, not ignored
            torch.func.jvp(fn, (x,), (x,))
        with pytest.raises(Exception):  # so is vmap
            torch.vmap(fn)(x[None])


def test_saved_tensor_hooks_see_the_saved_tensors():
    x, dy, w, b = norm_problem("rows", 2, 24, 35, "f32")
    x.requires_grad_(True)
    want = torch.autograd.grad(autograd.layer_norm(x, w, b), x, dy)[0]
    seen = []
    with torch.autograd.graph.saved_tensors_hooks(lambda v: (seen.append(v.shape), v)[1], lambda v: v.clone()):
        y = autograd.layer_norm(x, w, b)
    assert torch.equal(torch.autograd.grad(y, x, dy)[0], want) and len(seen) == 3


# ----------------------------------------------------------------------------
# refusals, on tensors that are where they would run
# ----------------------------------------------------------------------------

@pytest.mark.parametrize("call,match", [
    (lambda x, w: autograd.layer_norm(x.double(), w, w), "float32, bfloat16 or float16"),
    (lambda x, w: autograd.layer_norm(x, w.half(), w), "weight must be torch.float32"),
    (lambda x, w: autograd.layer_norm(x, w, w[:3]), "bias must have shape"),
    (lambda x, w: autograd.layer_norm(x, w, w, -1.0), "eps"),
    (lambda x, w: autograd.layer_norm(x, w, w, channel_dim=0), "from dimension"),
    (lambda x, w: autograd.layer_norm(x, w, w, channel_dim=-1, out_channel_dim=1), "from dimension"),
    (lambda x, w: autograd.layer_norm(w, w, w), "two dimensions"),
    (lambda x, w: autograd.layer_norm(x, w.cpu(), w), "GPU tensor"),
    (lambda x, w: autograd.scaled_residual(x.movedim(-1, 1), x.half(), w), "z must be torch.float32"),
    (lambda x, w: autograd.scaled_residual(x, x[:, :-1], w), "z must have shape"),
    (lambda x, w: autograd.scaled_residual(x.movedim(-1, 1), x, w, torch.ones(5, device=DEV)), "sample_scale must have"),
    (lambda x, w: autograd.scaled_residual(x.movedim(-1, 1), x, w, torch.ones(2, device=DEV, requires_grad=True)),
     "constant"),
])
def test_refusals(call, match):
    x, w = torch.zeros(2, 7, 6, device=DEV), torch.zeros(6, device=DEV)
    with pytest.raises(ValueError, match=match):
        call(x, w)


def test_second_derivatives_are_refused():
    x = torch.randn(2, 7, 6, device=DEV, requires_grad=True)
    for y in (autograd.layer_norm(x), autograd.scaled_residual(x, x.movedim(1, -1).contiguous())):
        g, = torch.autograd.grad((y * y).sum(), x, create_graph=True)
        with pytest.raises(RuntimeError):
            torch.autograd.grad(g.sum(), x)


def test_a_block_trains():
    """The operators together: a small network learns to tell gratings apart, with moments in 32 and in 8 bits."""
    from paper_2608_10805_amd import block

    for bits, dtype in ((32, torch.float32), (8, torch.float32), (8, torch.bfloat16)):
        losses = block.train(steps=60, state_bits=bits, dtype=dtype)
        assert sum(losses[-5:]) / 5 < 0.6 * losses[0], (bits, dtype, losses[0], losses[-5:])


@pytest.mark.parametrize("drop", [0.0, 0.5])
def test_the_block_is_the_formula(drop):
    """One block against the same steps in float64: y and every gradient, with the module's own drawn factors."""
    from paper_2608_10805_amd.block import WTConvNeXtBlock

    torch.manual_seed(1)
    m = WTConvNeXtBlock(12, levels=2, layer_scale=0.7, drop_path=drop, device=DEV)
    x = torch.randn(4, 12, 9, 10, device=DEV, requires_grad=True)
    rng = torch.cuda.get_rng_state(DEV)
    y = m(x)
    torch.cuda.set_rng_state(rng, DEV)
    keep = (torch.rand(4, device=DEV) >= drop).double() / (1 - drop)
    n = m.conv(x).double().movedim(1, -1)
    n = torch.nn.functional.layer_norm(n, (12,), m.norm.weight.double(), m.norm.bias.double(), 1e-6)
    z = torch.nn.functional.gelu(n @ m.expand.weight.double().T + m.expand.bias.double())
    z = z @ m.project.weight.double().T + m.project.bias.double()
    want = x.double() + (z * m.gamma.double() * keep.view(4, 1, 1, 1)).movedim(-1, 1)
    assert float((y - want).abs().max()) < 64 * 2.0 ** -24 * float(want.abs().max()) * 4
    names, ps = zip(*m.named_parameters())
    got = torch.autograd.grad(y, [x, *ps], torch.ones_like(y), retain_graph=True)
    ref_grads = torch.autograd.grad(want, [x, *ps], torch.ones_like(want))
    for name, a, b in zip(("x", *names), got, ref_grads):
        scale = float(b.abs().max())
        assert float((a.double() - b.double()).abs().max()) <= 2e-4 * scale + 1e-6, name
