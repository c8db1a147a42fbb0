"""Layer norm where the variance leaves float32's normal numbers."""
import pytest
import torch

from paper_2608_10805_amd import autograd, binding

from tests import _block as ref

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
LAYOUTS = {"rows": (-1, -1), "turned": (1, -1), "planes": (1, 1)}
# channels of the kernels that hold a pixel in registers (regular, irregular, many), and of those that sweep it again
CHANNELS = [8, 96, 100, 768, 5000]


def problem(layout, C, dtype, S=24):
    g = torch.Generator(device=DEV).manual_seed(C)
    cin, cout = LAYOUTS[layout]
    x = torch.randn((2, C, S) if cin == 1 else (2, S, C), generator=g, device=DEV)
    dy = torch.randn((2, C, S) if cout == 1 else (2, S, C), generator=g, device=DEV).to(ref.DTYPES[dtype])
    w, b = torch.rand(C, generator=g, device=DEV) + 0.5, torch.randn(C, generator=g, device=DEV)
    return x, dy, w, b


@pytest.mark.parametrize("layout", list(LAYOUTS))
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("C", CHANNELS)
def test_a_variance_that_overflows(layout, dtype, C):
    """Finite pixels near 1e20, whose squares are infinite: 1 / sqrt(inf) is 0, so y is the bias and dx is 0, and they
    add nothing to the weight's gradient. The other pixels keep their results."""
    cin, cout = LAYOUTS[layout]
    x, dy, w, b = problem(layout, C, dtype)
    pixels = x.movedim(cin, -1)  # (a view: [2, S, C])
    pixels[1, 7] = pixels[1, 7] * 1e20 + 3e20
    x = x.to(ref.DTYPES[dtype])
    y, mean, rstd = binding.layer_norm_forward(x, w, b, 1e-6, cin, cout)
    dx, dw, db = binding.layer_norm_backward(dy, x, mean, rstd, w, 1e-6, cin, cout)
    at = x.shape[2 if cin == 1 else 1] + 7
    assert float(rstd[at]) == 0.0 and int((rstd == 0).sum()) == 1
    y, dx = ref.to_rows(y, cout), ref.to_rows(dx, cin)
    assert torch.equal(y[at], b.to(ref.DTYPES[dtype]).double().cpu())
    assert bool((dx[at] == 0).all()) and bool(dx.isfinite().all()) and bool(y.isfinite().all())
    keep = torch.arange(len(y)) != at
    want, xhat, r = ref.norm(ref.to_rows(x, cin)[keep], w.double().cpu(), b.double().cpu(), 1e-6)
    ref.close(y[keep], want, dtype, 64 + C / 16)
    up = ref.to_rows(dy, cout)
    _, dweight, _ = ref.norm_grads(up[keep], xhat, r, w.double().cpu())
    ref.close(dw, dweight, "f32", 64, 8 * len(y) ** 0.5 + float(dweight.abs().max()))
    ref.close(db, up.sum(0), "f32", 64, 8 * len(y) ** 0.5 + float(up.sum(0).abs().max()))


@pytest.mark.parametrize("layout", list(LAYOUTS))
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("C", CHANNELS)
@pytest.mark.parametrize("power", [-47, -48, -49, -60, -63, -64, -65, -70, -73])
def test_a_variance_below_the_normal_numbers(layout, dtype, C, power):
    """An eps of 0 and channels of plus and minus a power of two: the mean is 0 and the variance the power's square,
    both exact down to 2^-149, so that y is plus and minus one to two roundings."""
    cin, cout = LAYOUTS[layout]
    x, _, w, b = problem(layout, C, dtype)
    sign = torch.ones(C, device=DEV)
    sign[1::2] = -1
    shape = (1, C, 1) if cin == 1 else (C,)
    x = (sign * 2.0 ** power).view(shape).expand(x.shape).to(ref.DTYPES[dtype]).contiguous()
    y, mean, rstd = binding.layer_norm_forward(x, None, None, 0.0, cin, cout)
    assert bool((mean == 0).all())
    assert float((rstd.double() * 2.0 ** power - 1).abs().max()) <= 2.0 ** -22
    ref.close(ref.to_rows(y, cout), sign.double().cpu().expand(48, C), dtype, 4)


@pytest.mark.parametrize("layout", list(LAYOUTS))
@pytest.mark.parametrize("C", [8, 100, 5000])
def test_a_constant_pixel_without_eps(layout, C):
    """A variance of 0 and an eps of 0: 0 * inf, as the formula has it; with an eps the bias."""
    x, _, w, b = problem(layout, C, "f32")
    one = torch.ones_like(x)
    assert bool(autograd.layer_norm(one, w, b, 0.0, *LAYOUTS[layout]).isnan().all())
    y = autograd.layer_norm(one, w, b, 2.0 ** -140, *LAYOUTS[layout])
    assert torch.equal(ref.to_rows(y, LAYOUTS[layout][1]), b.double().cpu().expand(48, C))
