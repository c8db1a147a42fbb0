"""Scaled residuals that the tiles' 32-bit offsets do not reach: the looping kernels."""
import pytest
import torch

from paper_2608_10805_amd import binding

from tests import _block as ref

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


def test_residual_of_planes_whose_offsets_pass_32_bits():
    """2^20 channels of 480 pixels (a tile and the image after it are 4 GB): both ends and every 997th channel, in
    full, against float64."""
    C, S = 1 << 20, 480
    g = torch.Generator(device=DEV).manual_seed(0)
    x = torch.empty(1, C, S, device=DEV).normal_(generator=g)
    z = torch.empty(1, S, C, device=DEV).normal_(generator=g)
    gamma = torch.empty(C, device=DEV).normal_(generator=g)
    keep = torch.tensor([1.25], device=DEV)
    some = torch.cat([torch.arange(0, C, 997), torch.arange(C - 70, C)]).unique()
    take = lambda t, dim: t.index_select(dim, some.to(DEV)).double().cpu()  # noqa: E731
    y = binding.scaled_residual_forward(x, z, gamma, keep)
    ref.close(take(y, 1), ref.residual(take(x, 1), take(z, 2), take(gamma, 0), keep.double().cpu()), "f32", 4, scale=32.0)
    del y
    dz, dgamma = binding.scaled_residual_backward(x, z, gamma, keep)  # x as dy
    want_dz, want_dgamma = ref.residual_grads(take(x, 1), take(z, 2), take(gamma, 0), keep.double().cpu())
    ref.close(take(dz, 2), want_dz, "f32", 4)
    ref.close(take(dgamma, 0), want_dgamma, "f32", 64, 8 * S ** 0.5 + float(want_dgamma.abs().max()))
    for need in ((True, False), (False, True)):
        again = binding.scaled_residual_backward(x, z, gamma, keep, *need)
        assert all(torch.equal(a, b) for a, b in zip(again, (dz, dgamma)) if a is not None)
    torch.cuda.empty_cache()


@pytest.mark.parametrize("C", [1, 2])
def test_residual_of_more_pixels_than_31_bits(C):
    """2^31 and some pixels of one and of two bfloat16 channels, every element. Small whole numbers and powers of two,
    so that all sums are exact in any order up to the last rounding."""
    S = (1 << 31) + 70 if C == 1 else (1 << 30) + 35
    B = C  # (two images of half the size)
    x = torch.empty(B, C, S, dtype=torch.bfloat16, device=DEV)
    z = torch.empty(B, S, C, dtype=torch.bfloat16, device=DEV)
    # patterns of different lengths along the pixels, so that a shift by a tile or an image shows
    at, step = torch.arange(7 * 5 * 64, device=DEV), 7 * 5 * 64
    for b in range(B):
        for c in range(C):
            for t, n, shift in ((x[b, c], 7, 3), (z[b, :, c], 5, 2)):
                wave = ((at + b + 2 * c) % n - shift).to(torch.bfloat16)
                whole = S // step * step
                t[:whole].view(-1, step).copy_(wave.expand(S // step, step)) if t.is_contiguous() else \
                    t[:whole].unflatten(0, (-1, step)).copy_(wave.expand(S // step, step))
                t[whole:].copy_(wave[:S - whole])
    gamma = torch.tensor([0.5, -2.0][:C], device=DEV)
    keep = torch.tensor([1.0, 4.0][:B], device=DEV)
    y = binding.scaled_residual_forward(x, z, gamma, keep)
    dz, dgamma = binding.scaled_residual_backward(x, z, gamma, keep)  # x as dy
    sums = [0.0] * C
    for b in range(B):
        for c in range(C):
            k = float(gamma[c] * keep[b])
            for i in range(0, S, 1 << 28):
                part = slice(i, min(S, i + (1 << 28)))
                px, pz = x[b, c, part].float(), z[b, part, c].float()
                # whole and half numbers below 32: exact in bfloat16
                assert torch.equal(y[b, c, part].float(), px + k * pz)
                assert torch.equal(dz[b, part, c].float(), k * px)
                sums[c] += float(keep[b]) * float((px * pz).sum(dtype=torch.float64))
    # terms of at most 24 in size, 2^31 of them in partial sums of a workgroup's own: in units of the sum of their sizes
    for c in range(C):
        assert abs(float(dgamma[c]) - sums[c]) <= 2.0 ** -24 * 2 * B * S * 24, c
    torch.cuda.empty_cache()
