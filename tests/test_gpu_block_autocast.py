"""The block and the network under torch.autocast."""
import pytest
import torch

from paper_2608_10805_amd.block import WTConvNeXt, WTConvNeXtBlock

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


@pytest.mark.parametrize("low", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
def test_the_block_under_autocast(low, dtype):
    """The products run in the lower type, the result and every gradient have the types they have without it, and
    differ by that type's rounding: in units of its half ulp, the products' inputs, weights and results, twice over,
    on a branch that is scaled by at most one."""
    torch.manual_seed(1)
    m = WTConvNeXtBlock(16, levels=1, layer_scale=1.0, device=DEV)
    x = torch.randn(2, 16, 12, 10, device=DEV).to(dtype).requires_grad_(True)
    dy = torch.randn(x.shape, device=DEV).to(dtype)
    names, ps = zip(*m.named_parameters())
    runs = []
    for on in (False, True):
        with torch.autocast("cuda", dtype=low, enabled=on):
            y = m(x)
        runs.append((y.detach(), *torch.autograd.grad(y, [x, *ps], dy)))
    for name, a, b in zip(("y", "x", *names), *runs):
        assert a.dtype == b.dtype and a.shape == b.shape, name
        room = 16 * max(torch.finfo(low).eps, torch.finfo(dtype).eps) * float(a.float().abs().max()) + 1e-6
        assert float((a.float() - b.float()).abs().max()) <= room, name


def test_the_network_trains_under_autocast():
    torch.manual_seed(0)
    model = WTConvNeXt(drop_path=0.1, device=DEV)
    images, label = torch.randn(4, 3, 64, 64, device=DEV), torch.arange(4, device=DEV)
    with torch.autocast("cuda", dtype=torch.bfloat16):
        loss = torch.nn.functional.cross_entropy(model(images), label)
    loss.backward()
    assert bool(loss.isfinite())
    assert all(p.grad is not None and bool(p.grad.isfinite().all()) for p in model.parameters())
