"""Host-side checks of the operators around the convolution (no GPU): the C
entry points refuse bad arguments before any HIP call, and the binding refuses
tensors that do not fit before any library call."""
import ctypes

import pytest

torch = pytest.importorskip("torch")

from paper_2608_10805_amd import autograd, binding, optim  # noqa: E402

OK, NULL, SHAPE, DTYPE, ALIAS, WORKSPACE, UNSUPPORTED = 0, 1, 2, 5, 6, 7, 8
A = [(i + 1) << 40 for i in range(10)]  # addresses that are never dereferenced


def norm(B=2, S=49, C=96, cin=1, cout=0, xs=0, ds=0, eps=1e-6, dtype=0):
    return binding.NormDesc(B, S, C, cin, cout, xs, ds, eps, dtype)


@pytest.mark.parametrize("change,code", [
    (dict(B=-1), SHAPE), (dict(S=-1), SHAPE), (dict(C=0), SHAPE), (dict(C=(1 << 20) + 1), SHAPE),
    (dict(B=1 << 40, S=1 << 40), SHAPE), (dict(B=1, S=1 << 45), SHAPE), (dict(dtype=3), DTYPE),
    (dict(cin=0, cout=1), UNSUPPORTED), (dict(cin=2), UNSUPPORTED), (dict(cout=5), UNSUPPORTED),
    (dict(eps=-1.0), UNSUPPORTED), (dict(eps=float("nan")), UNSUPPORTED), (dict(eps=float("inf")), UNSUPPORTED),
    (dict(xs=96), SHAPE), (dict(cin=0, xs=95), SHAPE), (dict(ds=95), SHAPE), (dict(cin=0, xs=1 << 60), SHAPE),
    (dict(cout=1, ds=96), SHAPE),
])
def test_norm_descriptors(change, code):
    d = norm(**change)
    assert binding.wtconv_layer_norm_forward(d, A[0], A[1], A[2], A[3], A[4], A[5], None) == code
    assert binding.wtconv_layer_norm_backward_workspace_bytes(d) == 0
    assert binding.wtconv_layer_norm_backward(d, A[0], A[1], A[2], A[3], A[4], A[5], A[6], A[7], A[8], 1 << 30,
                                              None) == code


def test_norm_arguments():
    f = lambda *p: binding.wtconv_layer_norm_forward(norm(), *p, None)  # noqa: E731
    assert f(None, A[1], A[2], A[3], A[4], A[5]) == NULL
    assert f(A[0], A[1], A[2], None, A[4], A[5]) == NULL
    assert f(A[0], A[1], A[2], A[3], A[4], None) == NULL
    assert f(A[0], A[1], A[2], A[0] + 64, A[4], A[5]) == ALIAS
    assert f(A[0], A[3] + 128, A[2], A[3], A[4], A[5]) == ALIAS
    assert f(A[0], A[1], A[2], A[3], A[4], A[4] + 8) == ALIAS
    assert f(A[0] + 2, A[1], A[2], A[3], A[4], A[5]) == SHAPE
    assert binding.load().wtconv_layer_norm_forward(None, A[0], None, None, A[3], None, None, None) == NULL
    need = binding.wtconv_layer_norm_backward_workspace_bytes(norm())
    assert need > 0 and need % 256 == 0
    g = lambda ws=A[8], size=need, dx=A[5], dw=A[6], x=A[1]: binding.wtconv_layer_norm_backward(  # noqa: E731
        norm(), A[0], x, A[2], A[3], A[4], dx, dw, A[7], ws, size, None)
    assert g(ws=None) == WORKSPACE and g(size=need - 1) == WORKSPACE and g(ws=A[8] + 8) == WORKSPACE
    assert g(dx=A[1]) == ALIAS and g(dw=A[7]) == ALIAS and g(ws=A[0] + 256) == ALIAS and g(x=None) == NULL
    assert binding.wtconv_layer_norm_backward(norm(), A[0], A[1], A[2], A[3], A[4], None, None, None, None, 0,
                                              None) == OK  # nothing is asked for
    assert binding.wtconv_layer_norm_forward(norm(B=0), None, None, None, None, None, None, None) == OK


def test_residual_arguments():
    d = binding.ResidualDesc(2, 49, 96, 0)
    f = lambda desc=d, x=A[0], z=A[1], y=A[4]: binding.wtconv_scaled_residual_forward(  # noqa: E731
        desc, x, z, A[2], A[3], y, None)
    assert f(binding.ResidualDesc(2, 49, 0, 0)) == SHAPE and f(binding.ResidualDesc(2, 49, 96, 9)) == DTYPE
    assert f(binding.ResidualDesc(-2, 49, 96, 0)) == SHAPE
    assert f(x=None) == NULL and f(z=None) == NULL and f(y=None) == NULL
    assert f(y=A[0]) == ALIAS and f(y=A[1] + 64) == ALIAS and f(z=A[1] + 1) == SHAPE
    assert f(binding.ResidualDesc(0, 49, 96, 0), x=None) == OK
    need = binding.wtconv_scaled_residual_backward_workspace_bytes(d)
    assert need > 0
    g = lambda z=A[1], dz=A[4], dg=A[5], ws=A[6], size=need: binding.wtconv_scaled_residual_backward(  # noqa: E731
        d, A[0], z, A[2], A[3], dz, dg, ws, size, None)
    assert g(z=None) == NULL and g(ws=None) == WORKSPACE and g(size=need - 1) == WORKSPACE
    assert g(dz=A[0] + 64) == ALIAS and g(dg=A[4] + 4) == ALIAS
    assert g(dz=None, dg=None, z=None) == OK


def adamw(group={}, tensor={}, dtype=0, bits=32, scale=None):
    g = dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.0, step=1, key=0, exp_avg=A[2], exp_avg_sq=A[3],
             exp_avg_scale=A[4], exp_avg_sq_scale=A[5])
    t = dict(param=A[0], grad=A[1], numel=100, offset=64, group=0)
    return binding.wtconv_adamw_step([binding.AdamWGroup(**{**g, **group})], [binding.AdamWTensor(**{**t, **tensor})],
                                     dtype, bits, scale, None)


@pytest.mark.parametrize("change,code", [
    (dict(group=dict(lr=-1.0)), UNSUPPORTED), (dict(group=dict(beta1=1.0)), UNSUPPORTED),
    (dict(group=dict(beta2=-0.1)), UNSUPPORTED), (dict(group=dict(eps=float("nan"))), UNSUPPORTED),
    (dict(group=dict(weight_decay=float("inf"))), UNSUPPORTED), (dict(group=dict(step=0)), UNSUPPORTED),
    (dict(group=dict(exp_avg=None)), NULL), (dict(group=dict(exp_avg_scale=None), bits=8), NULL),
    (dict(group=dict(exp_avg_sq=A[3] + 4)), SHAPE), (dict(tensor=dict(param=None)), NULL),
    (dict(tensor=dict(grad=None)), NULL), (dict(tensor=dict(numel=-1)), SHAPE), (dict(tensor=dict(offset=32)), SHAPE),
    (dict(tensor=dict(offset=-64)), SHAPE), (dict(tensor=dict(group=1)), SHAPE), (dict(tensor=dict(group=-1)), SHAPE),
    (dict(tensor=dict(param=A[0] + 2)), SHAPE), (dict(tensor=dict(grad=A[0] + 64)), ALIAS), (dict(dtype=4), DTYPE),
    (dict(bits=16), UNSUPPORTED), (dict(scale=A[6] + 1), SHAPE), (dict(tensor=dict(numel=1 << 50)), SHAPE),
    (dict(tensor=dict(numel=0, param=None)), OK),
])
def test_adamw_arguments(change, code):
    assert adamw(**change) == code


def test_adamw_moments_arguments():
    f = lambda n=128, m=A[0], out=A[4], dtype=1: binding.wtconv_adamw_moments(  # noqa: E731
        n, m, A[1], A[2], A[3], out, A[5], dtype, None)
    assert f(n=100) == SHAPE and f(n=-64) == SHAPE and f(m=None) == NULL and f(dtype=7) == DTYPE
    assert f(out=A[4] + 8) == SHAPE and f(out=A[0]) == ALIAS and f(n=0, m=None) == OK


def test_struct_layouts():
    assert ctypes.sizeof(binding.NormDesc) == 64 and ctypes.sizeof(binding.ResidualDesc) == 24
    assert ctypes.sizeof(binding.AdamWGroup) == 88 and ctypes.sizeof(binding.AdamWTensor) == 40


def desc(x, **kw):
    return binding.norm_desc(x, on_gpu=False, **kw)


def test_norm_problems():
    x = torch.zeros(2, 6, 5, 7)
    d, shape = desc(x, channel_dim=1)
    assert (d.B, d.S, d.C, d.in_, d.out, shape) == (2, 35, 6, 1, 1, (2, 6, 5, 7))
    d, shape = desc(x, channel_dim=1, out_channel_dim=-1, dy=torch.zeros(2, 5, 7, 6))
    assert (d.in_, d.out, d.dy_stride, shape) == (1, 0, 6, (2, 5, 7, 6))
    d, shape = desc(x, weight=torch.ones(7))
    assert (d.B, d.S, d.C, d.x_stride, shape) == (2, 30, 7, 7, (2, 6, 5, 7))
    d, _ = desc(torch.zeros(4, 9, 20)[..., 3:9])
    assert (d.B, d.S, d.C, d.x_stride) == (4, 9, 6, 20)
    d, _ = desc(torch.zeros(4, 9, 20)[:, :1, 3:9])  # one row of each image
    assert (d.B, d.S, d.x_stride) == (4, 1, 180)
    d, _ = desc(torch.zeros(0, 9, 6))
    assert (d.B, d.S, d.C) == (0, 0, 6)
    d, _ = desc(torch.zeros(2, 6), channel_dim=1)
    assert (d.B, d.S, d.C) == (2, 1, 6)


@pytest.mark.parametrize("call,match", [
    (lambda x: desc(x[:, :, :4]), "one distance"),
    (lambda x: desc(x.transpose(2, 3)), "one distance"),
    (lambda x: desc(x[..., ::2]), "one distance"),
    (lambda x: desc(x[..., :1].expand(2, 6, 5, 7)), "one distance"),
    (lambda x: desc(x[0, 0, 0].expand(4, 7)), "one distance"),
    (lambda x: desc(x[:, ::2], channel_dim=1), "contiguous"),
    (lambda x: desc(x.int()), "float32, bfloat16 or float16"),
    (lambda x: desc(x[0, 0, 0]), "two dimensions"),
    (lambda x: desc(x[..., :0]), "channels must be"),
    (lambda x: desc(x, channel_dim=2), "from dimension"),
    (lambda x: desc(x, weight=torch.ones(6)), "weight must have shape"),
    (lambda x: desc(x, bias=torch.ones(7).double()), "bias must be"),
    (lambda x: desc(x, eps="1"), "eps"),
    (lambda x: desc(x, dy=x.half()), "dy must be"),
    (lambda x: desc(x, dy=x[:1]), "dy must be"),
    (lambda x: desc(x, dy=torch.ones(1).expand(2, 6, 5, 7)), "dy must be contiguous"),
    (lambda x: binding.residual_desc(x, x, on_gpu=False), "z must have shape"),
    (lambda x: binding.residual_desc(x.half(), torch.zeros(2, 5, 7, 6), on_gpu=False), "z must be"),
    (lambda x: binding.residual_desc(x, torch.zeros(2, 5, 7, 6), torch.ones(5), on_gpu=False), "gamma must have"),
    (lambda x: binding.residual_desc(x[:, ::2], torch.zeros(2, 5, 7, 3), on_gpu=False), "x must be contiguous"),
])
def test_problems_that_are_refused(call, match):
    with pytest.raises(ValueError, match=match):
        call(torch.zeros(2, 6, 5, 7))


def test_entry_points_refuse_host_tensors():
    x, w = torch.zeros(2, 6, 5), torch.ones(5)
    for call in (lambda: autograd.layer_norm(x, w, w), lambda: autograd.layer_norm(x, channel_dim=1),
                 lambda: autograd.scaled_residual(x, x.movedim(1, -1)), lambda: binding.layer_norm_forward(x),
                 lambda: binding.layer_norm_backward(x, x, w, w), lambda: binding.scaled_residual_backward(x, x),
                 lambda: optim.AdamW([torch.nn.Parameter(x)])):
        with pytest.raises(ValueError, match="GPU tensor"):
            call()
    with pytest.raises(ValueError, match="must be a tensor"):
        autograd.layer_norm([1.0, 2.0])


def test_a_residual_needs_its_branch():
    with pytest.raises(ValueError, match="z"):
        binding.scaled_residual_forward(torch.zeros(2, 3, 4), None)
    with pytest.raises(ValueError, match="z"):
        binding.scaled_residual_backward(torch.zeros(2, 3, 4), None)


def test_rounding_keys_differ():
    """The key of each step, group and seed is another one (of 2^32; 20000 of them share about 0.05 pairs)."""
    keys = {optim.rounding_key(seed, step, group) for seed in range(5) for step in range(1000) for group in range(4)}
    assert len(keys) >= 19998


def test_code_tables_cover_a_block():
    """The codes rise, start at 0, have three mantissa bits, and the top exponent is only reached by rounding up."""
    from tests import _block as ref

    for bits in (4, 5):
        v = ref.code_values(bits)
        assert v[0] == 0 and bool((v[1:] > v[:-1]).all()) and float(v[8]) == 2.0
        assert float(v[(2 ** bits - 2) * 8]) == 2.0 ** (2 ** bits - 2) and len(v) == 2 ** (bits + 3)


def test_formulas_against_differences():
    """The references' gradients against central differences of the references, in float64."""
    from tests import _block as ref

    g = torch.Generator().manual_seed(0)
    r = lambda *s: torch.randn(s, generator=g, dtype=torch.float64)  # noqa: E731
    x, w, b, dy = r(4, 6), r(6), r(6), r(4, 6)
    y, xhat, rstd = ref.norm(x, w, b, 1e-3)
    grads = ref.norm_grads(dy, xhat, rstd, w)
    f = lambda: float((ref.norm(x, w, b, 1e-3)[0] * dy).sum())  # noqa: E731
    p, z, gamma, keep, up = r(2, 3, 4), r(2, 4, 3), r(3), r(2), r(2, 3, 4)
    dz, dgamma = ref.residual_grads(up, z, gamma, keep)
    h = lambda: float((ref.residual(p, z, gamma, keep) * up).sum())  # noqa: E731
    for fn, pairs in ((f, ((x, grads[0]), (w, grads[1]), (b, grads[2]))), (h, ((z, dz), (gamma, dgamma)))):
        for t, want in pairs:
            flat = t.view(-1)
            for i in range(flat.numel()):
                old = float(flat[i])
                flat[i] = old + 1e-5
                hi = fn()
                flat[i] = old - 1e-5
                lo = fn()
                flat[i] = old
                assert abs((hi - lo) / 2e-5 - float(want.reshape(-1)[i])) < 1e-7
