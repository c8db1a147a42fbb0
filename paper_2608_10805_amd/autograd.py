"""torch.autograd wrappers and nn.Modules around the fused WTConv library: the
convolution, and the layer norm and scaled residual of the block around it.

Of the convolution, only x and the parameters are saved for backward (no
per-level subband tensors): the backward kernel recomputes both Haar pyramids
on chip. The layer norm saves x and two floats a pixel.
"""
import ctypes
import math

import torch

from . import binding


class WTConvFunction(torch.autograd.Function):
    """y = WTConv(x; base_w, base_scale, base_bias, level_w[0..L-1], level_scale[0..L-1]),
    base_bias optional (None)."""

    @staticmethod
    def forward(ctx, x, base_w, base_scale, base_bias, *level_params):
        L = len(level_params) // 2
        level_w, level_scale = list(level_params[:L]), list(level_params[L:])
        x = x.contiguous()
        y = binding.forward(x, base_w, base_scale, level_w, level_scale, bias=base_bias)
        ctx.save_for_backward(x, base_w, base_scale, base_bias, *level_params)
        return y

    @staticmethod
    def backward(ctx, dy):
        x, base_w, base_scale, base_bias, *level_params = ctx.saved_tensors
        return _backward(x, dy, base_w, base_scale, base_bias, level_params, ctx.needs_input_grad[0],
                         base_bias is not None and ctx.needs_input_grad[3])


def _backward(x, dy, base_w, base_scale, base_bias, level_params, need_dx, need_dbias):
    L = len(level_params) // 2
    out = binding.backward(x, dy.contiguous(), base_w, base_scale, level_params[:L], level_params[L:],
                           need_dx=need_dx, bias=base_bias, need_dbias=need_dbias)
    dx, dbw, dbs, dlw, dls = out[:5]
    return (dx, dbw, dbs, out[5] if need_dbias else None, *dlw, *dls)


_native = None


def _load_native(x=None):
    """The native host path (csrc/wtconv_torch.cpp), given the library's entry
    points; False where it was not built, and for an x that is no GPU tensor
    (nothing is loaded for it)."""
    global _native
    if x is not None and not (isinstance(x, torch.Tensor) and x.is_cuda):
        return False
    if _native is None:
        try:
            from . import _wtconv_torch as ext
        except ImportError:
            _native = False
        else:
            lib = binding.load()
            ext.init(*(ctypes.cast(getattr(lib, n), ctypes.c_void_p).value
                       for n in ("wtconv_forward_workspace_bytes", "wtconv_forward",
                                 "wtconv_backward_workspace_bytes", "wtconv_backward")), _backward)
            _native = ext
    return _native


def wtconv(x, base_w, base_scale, level_w, level_scale, base_bias=None):
    """The operator under autograd. The plain case (dense, contiguous GPU tensors
    that fit the problem and override no torch function, nothing tracing or
    transforming) runs from native code; WTConvFunction does the same for every
    other one, or raises."""
    level_w, level_scale = tuple(level_w), tuple(level_scale)  # (any iterable)
    ext = _native if _native is not None else _load_native(x)
    if ext and len(level_w) == len(level_scale) and not torch.compiler.is_compiling():
        y = ext.apply(x, base_w, base_scale, base_bias, level_w + level_scale)
        if y is not None:
            return y
    return WTConvFunction.apply(x, base_w, base_scale, base_bias, *level_w, *level_scale)


class WTConv2d(torch.nn.Module):
    """Drop-in depthwise replacement: k x k base conv plus an L-level Haar branch.

    Parameters are float32 whatever the activation dtype. Initialisation follows
    the synthetic recipe of the tests (uniform kernels, base scale 1, small
    level scales) and can be overwritten freely.
    """

    def __init__(self, channels: int, kernel_size: int = 5, levels: int = 1, bias: bool = False, device=None):
        super().__init__()
        C, k = channels, kernel_size
        bound = 1.0 / math.sqrt(k * k)
        self.base_w = torch.nn.Parameter(torch.empty(C, k, k, device=device).uniform_(-bound, bound))
        self.base_scale = torch.nn.Parameter(torch.ones(C, device=device))
        self.base_bias = torch.nn.Parameter(torch.zeros(C, device=device)) if bias else None
        self.level_w = torch.nn.ParameterList(
            [torch.nn.Parameter(torch.empty(4 * C, k, k, device=device).uniform_(-bound, bound))
             for _ in range(levels)])
        self.level_scale = torch.nn.ParameterList(
            [torch.nn.Parameter(torch.full((4 * C,), 0.1, device=device)) for _ in range(levels)])

    def forward(self, x):
        return wtconv(x, self.base_w, self.base_scale, list(self.level_w), list(self.level_scale), self.base_bias)


_block = None


def load_block(x):
    """The native host path of the operators around the convolution (csrc_block/block_torch.cpp), given the library's
    entry points; False where it was not built, and for an x that is no GPU tensor (nothing is loaded for it)."""
    global _block
    if not (isinstance(x, torch.Tensor) and x.is_cuda):
        return False
    if _block is None:
        try:
            from . import _wtconv_block as ext
        except ImportError:
            _block = False
        else:
            lib = binding.load()
            ext.init([ctypes.cast(getattr(lib, n), ctypes.c_void_p).value
                      for n in ("wtconv_layer_norm_forward", "wtconv_layer_norm_backward_workspace_bytes",
                                "wtconv_layer_norm_backward", "wtconv_scaled_residual_forward",
                                "wtconv_scaled_residual_backward_workspace_bytes", "wtconv_scaled_residual_backward",
                                "wtconv_adamw_step", "wtconv_adamw_moments")], _norm_backward, _residual_backward)
            _block = ext
    return _block


class _Made(torch.autograd.Function):
    """A gradient as a result of what it was made of, so that a gradient of it reaches this error."""

    @staticmethod
    def forward(ctx, grad, *sources):
        return grad.detach()

    @staticmethod
    def backward(ctx, _):
        raise RuntimeError("the operators around the convolution cannot be differentiated twice")


def _made_of(grad, *sources):
    """A gradient that a backward pass was asked for, or None: with create_graph it depends on its sources (tensors or
    None) that need gradients, and differentiating it is refused rather than taken for zero."""
    if grad is None or not torch.is_grad_enabled() or not any(t is not None and t.requires_grad for t in sources):
        return grad
    return _Made.apply(grad, *sources)


def _dense_rows(t):
    return t if binding._row_stride(t) is not None else t.contiguous()


class LayerNormFunction(torch.autograd.Function):
    """layer_norm() of tensors as binding.norm_desc takes them."""

    @staticmethod
    def forward(ctx, x, weight, bias, eps, channel_dim, out_channel_dim):
        y, mean, rstd = binding.layer_norm_forward(x, weight, bias, eps, channel_dim, out_channel_dim)
        ctx.save_for_backward(x, mean, rstd, weight)
        ctx.args = (eps, channel_dim, out_channel_dim)
        return y

    @staticmethod
    def backward(ctx, dy):
        return (*_norm_backward((*ctx.args, *ctx.needs_input_grad[:3]), dy, *ctx.saved_tensors), None, None, None)


def _norm_backward(args, dy, x, mean, rstd, weight):
    """args: eps, the two channel dimensions and which gradients are asked for."""
    with torch.no_grad():
        rows = _dense_rows(dy) if args[2] == -1 else dy.contiguous()
        dx, dweight, dbias = binding.layer_norm_backward(rows, x, mean, rstd, weight, *args)
    return _made_of(dx, dy, x, weight), _made_of(dweight, dy, x), _made_of(dbias, dy)


def layer_norm(x, weight=None, bias=None, eps=1e-6, channel_dim=-1, out_channel_dim=None):
    """Layer norm over the channels of every pixel, under autograd:
    (x - mean) / sqrt(variance + eps) * weight + bias.

    The channels are dimension `channel_dim` of x, the last (-1: rows, x [..., C]) or dimension 1 (planes, x [B, C,
    ...]), and dimension `out_channel_dim` of the result (by default the same one; 1 can be moved to -1, so that the
    pointwise products that follow find the channels adjacent). x is float32, bfloat16 or float16, weight and bias
    [C] float32 or None; sums are float32.
    """
    if out_channel_dim is None:
        out_channel_dim = channel_dim
    ext = _block if _block is not None else load_block(x)
    if ext and not torch.compiler.is_compiling():
        y = ext.layer_norm(x, weight, bias, eps, channel_dim, out_channel_dim)
        if y is not None:
            return y
    if channel_dim == 1 and isinstance(x, torch.Tensor) and x.dim() > 2 and not x.is_contiguous():
        rows = x.movedim(1, -1)
        if binding._row_stride(rows) is not None:  # planes held as rows (channels_last) are normalised as they lie
            y = layer_norm(rows, weight, bias, eps)
            return y if out_channel_dim == -1 else y.movedim(-1, 1)
    if isinstance(x, torch.Tensor) and x.dim() > 1:
        x = x.contiguous() if channel_dim == 1 else _dense_rows(x)
    return LayerNormFunction.apply(x, weight, bias, eps, channel_dim, out_channel_dim)


class ScaledResidualFunction(torch.autograd.Function):
    """scaled_residual() of contiguous tensors."""

    @staticmethod
    def forward(ctx, x, z, gamma, sample_scale):
        y = binding.scaled_residual_forward(x, z, gamma, sample_scale)
        # z is needed for the gradient of gamma alone
        ctx.save_for_backward(z if ctx.needs_input_grad[2] else None, gamma, sample_scale)
        return y

    @staticmethod
    def backward(ctx, dy):
        return (*_residual_backward(ctx.needs_input_grad[:3], dy, *ctx.saved_tensors), None)


def _residual_backward(need, dy, z, gamma, sample_scale):
    """need: which of the gradients of x, z and gamma are asked for."""
    with torch.no_grad():
        dz, dgamma = binding.scaled_residual_backward(dy.contiguous(), z, gamma, sample_scale, *need[1:])
    return dy if need[0] else None, _made_of(dz, dy, gamma), _made_of(dgamma, dy, z)


def scaled_residual(x, z, gamma=None, sample_scale=None):
    """x + sample_scale * gamma * z under autograd, where x [B, C, ...] and the result are planes and z [B, ..., C]
    is rows, as the pointwise products leave them. gamma: [C] float32, the layer scale; sample_scale: [B] float32,
    one factor an image (0 where stochastic depth drops the branch), a constant for autograd. None means ones."""
    ext = _block if _block is not None else load_block(x)
    if ext and not torch.compiler.is_compiling():
        y = ext.scaled_residual(x, z, gamma, sample_scale)
        if y is not None:
            return y
    if isinstance(sample_scale, torch.Tensor) and sample_scale.requires_grad:
        raise ValueError("sample_scale is a constant: it has no gradient")
    if isinstance(x, torch.Tensor) and isinstance(z, torch.Tensor):
        x, z = x.contiguous(), z.contiguous()
    return ScaledResidualFunction.apply(x, z, gamma, sample_scale)


class LayerNorm(torch.nn.Module):
    """layer_norm() with its parameters, float32 whatever the activation dtype."""

    def __init__(self, channels: int, eps: float = 1e-6, channel_dim: int = -1, out_channel_dim=None, device=None):
        super().__init__()
        self.weight = torch.nn.Parameter(torch.ones(channels, device=device))
        self.bias = torch.nn.Parameter(torch.zeros(channels, device=device))
        self.eps, self.channel_dim, self.out_channel_dim = eps, channel_dim, out_channel_dim

    def forward(self, x):
        return layer_norm(x, self.weight, self.bias, self.eps, self.channel_dim, self.out_channel_dim)
