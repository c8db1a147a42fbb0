"""Float64 references of the operators around the convolution, on the CPU, and
the bounds that their results are held to."""
import math

import torch

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
# Half a unit in the last place of the storage type, relative: what rounding the
# exact result once costs (2^-24, 2^-8, 2^-11). float32 results also carry the
# sums' own rounding.
HALF_ULP = {k: torch.finfo(t).eps / 2 for k, t in DTYPES.items()}


def close(got, want, dtype, sums=64, scale=None):
    """Every element within the storage type's rounding of its own size and `sums` float32 roundings of `scale` (by
    default the largest reference value), which is how far sums of that many terms are off at worst."""
    got, want = got.detach().double().cpu(), want.double()
    assert got.shape == want.shape, (got.shape, want.shape)
    if want.numel() == 0:
        return
    scale = float(want.abs().max()) if scale is None else scale
    tiny = 2.0 ** -24 if dtype == "f16" else 2.0 ** -133 if dtype == "bf16" else 2.0 ** -149
    room = HALF_ULP[dtype] * want.abs() * 1.01 + sums * 2.0 ** -24 * scale + tiny
    off = (got - want).abs()
    assert bool((off <= room).all()), f"off by {float((off / room).max()):.2f} of the bound"


def norm(x, w, b, eps):
    """x [pixels, C] in float64: y, xhat, rstd."""
    mean = x.mean(1, keepdim=True)
    rstd = 1 / torch.sqrt(((x - mean) ** 2).mean(1, keepdim=True) + eps)
    xhat = (x - mean) * rstd
    y = xhat * (w if w is not None else 1.0) + (b if b is not None else 0.0)
    return y, xhat, rstd


def norm_grads(dy, xhat, rstd, w):
    g = dy * (w if w is not None else 1.0)
    dx = rstd * (g - g.mean(1, keepdim=True) - xhat * (g * xhat).mean(1, keepdim=True))
    return dx, (dy * xhat).sum(0), dy.sum(0)


def to_rows(t, channel_dim):
    """[pixels, C] in float64 on the CPU."""
    t = t.detach().double().cpu()
    t = t.movedim(1, -1) if channel_dim == 1 else t
    return t.reshape(-1, t.shape[-1])


def from_rows(rows, shape, channel_dim):
    """The inverse of to_rows for a tensor of that shape."""
    if channel_dim == -1:
        return rows.reshape(shape)
    return rows.reshape(shape[0], *shape[2:], shape[1]).movedim(-1, 1)


def residual(x, z, gamma, keep):
    C, B = x.shape[1], x.shape[0]
    scale = gamma if gamma is not None else torch.ones(C, dtype=torch.float64)
    k = keep if keep is not None else torch.ones(B, dtype=torch.float64)
    return x + (z * scale * k.view(-1, *[1] * (z.dim() - 1))).movedim(-1, 1)


def residual_grads(dy, z, gamma, keep):
    C, B = dy.shape[1], dy.shape[0]
    scale = gamma if gamma is not None else torch.ones(C, dtype=torch.float64)
    k = (keep if keep is not None else torch.ones(B, dtype=torch.float64)).view(-1, *[1] * (dy.dim() - 1))
    rows = dy.movedim(1, -1) * k
    return rows * scale, (rows * z).reshape(-1, C).sum(0)


def adamw(p, g, m, v, t, lr, betas, eps, decay):
    b1, b2 = betas
    m = b1 * m + (1 - b1) * g
    v = b2 * v + (1 - b2) * g * g
    p = p * (1 - lr * decay) - lr / (1 - b1 ** t) * m / (v.sqrt() / math.sqrt(1 - b2 ** t) + eps)
    return p, m, v


def code_values(exponent_bits):
    """What the codes 0 to 2^(exponent_bits + 3) - 1 stand for under the scale 127 + 0, times 2^top: a float of that
    many exponent bits and three mantissa bits, its smallest ones subnormal."""
    out = []
    for c in range(1 << (exponent_bits + 3)):
        field, mantissa = c >> 3, c & 7
        out.append((1 + mantissa / 8) * 2.0 ** field if field else mantissa / 4)
    return torch.tensor(out, dtype=torch.float64)


def decode(codes, scales, signed):
    """Float64 values of 8-bit codes (a whole number of blocks of 64)."""
    top = 14 if signed else 30
    table = code_values(4 if signed else 5)
    c = codes.cpu().long()
    sign = torch.where(c >= 128, -1.0, 1.0).double() if signed else torch.ones(c.shape, dtype=torch.float64)
    size = table[c & 127] if signed else table[c]
    return sign * size * (2.0 ** (scales.cpu().double() - 127 - top)).repeat_interleave(64)
