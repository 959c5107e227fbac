"""Torch front doors to layer norm: `layer_norm(x, weight, bias)`, one fq_norm_forward and one fq_norm_backward call, and `layer_norm_int8`,
whose codes and scales `linear_int8` takes.

Marshalling only; torch owns the memory (outputs and the backward workspace come from its caching allocator) and the stream (the current
one).  There is no CPU path: CPU tensors raise.
"""
import torch
from torch.autograd import forward_ad
from torch.autograd.function import once_differentiable

from . import binding as fq


def _rows(t, width):
    """t as a matrix of rows of `width` values, without a copy where rows lie one distance apart."""
    t = t.reshape(-1, width) if width else t.reshape(t.shape[:-1].numel(), 0)
    if (width > 1 and t.stride(1) != 1) or (t.shape[0] > 1 and t.stride(0) < width):
        t = t.contiguous()
    return t


def _check(x, weight, bias):
    if not x.is_cuda:
        raise RuntimeError("layer_norm runs on the GPU only (no CPU fallback)")
    if x.dim() < 1:
        raise ValueError("x must have a dimension to normalise")
    for t, name in ((weight, "weight"), (bias, "bias")):
        if t is not None and tuple(t.shape) != (x.shape[-1],):
            raise ValueError("%s must have %d values" % (name, x.shape[-1]))


class _LayerNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, eps, out_dtype):
        _check(x, weight, bias)
        width = x.shape[-1]
        x2 = _rows(x, width)
        y = torch.empty(x.shape, dtype=out_dtype or x.dtype, device=x.device)
        stats = torch.empty((x2.shape[0], 2), dtype=torch.float32, device=x.device) if any(ctx.needs_input_grad) else None
        with torch.cuda.device(x.device):
            fq.fq_norm_forward(fq.FqNorm.from_torch(
                x2, y=y.view(x2.shape), weight=None if weight is None else weight.contiguous(),
                bias=None if bias is None else bias.contiguous(), stats=stats, eps=eps))
        # (the bias is saved for its type alone)
        ctx.save_for_backward(x, weight, stats)
        ctx.meta = eps, bias is not None, None if bias is None else bias.dtype
        return y

    @staticmethod
    @once_differentiable
    def backward(ctx, gy):
        x, weight, stats = ctx.saved_tensors
        eps, has_bias, bias_dtype = ctx.meta
        want_x, want_w, want_b = ctx.needs_input_grad[:3]
        width = x.shape[-1]
        x2 = _rows(x, width)
        g2 = _rows(gy, width)
        gx = torch.empty(x.shape, dtype=x.dtype, device=x.device) if want_x else None
        gw = torch.empty(width, dtype=weight.dtype, device=x.device) if want_w else None
        gb = torch.empty(width, dtype=bias_dtype, device=x.device) if want_b else None
        with torch.cuda.device(x.device):
            d = fq.FqNorm.from_torch(x2, weight=None if weight is None else weight.contiguous(), stats=stats, gy=g2,
                                     gx=None if gx is None else gx.view(x2.shape), gweight=gw, gbias=gb, eps=eps)
            # A fresh workspace per call keeps concurrent streams apart.
            workspace = torch.empty(fq.fq_norm_workspace_bytes(d), dtype=torch.uint8, device=x.device)
            fq.fq_norm_backward(d, workspace)
        return gx, gw, gb, None, None


def layer_norm(x, weight=None, bias=None, eps=1e-5, out_dtype=None):
    """y = (x - mean) / sqrt(var + eps) * weight + bias over the last dimension.

    x: float16 or float32; weight, bias: one value per place of the last dimension, both float16 or both float32, or None.
    out_dtype: float16 or float32 (default: x's).  Differentiable with respect to x, weight and bias, once; the sums of a row are
    binary64, and nothing is saved but references to x and weight and two floats a row.
    """
    return _LayerNorm.apply(x, weight, bias, float(eps), out_dtype)


def layer_norm_int8(x, weight=None, bias=None, eps=1e-5):
    """(codes, scales) of `layer_norm(x, weight, bias, eps)` in one launch: int8 codes of x's shape and a float32 scale per row, as
    `linear_int8(codes, w, w_scale, x_scale=scales.flatten())` takes them.  No gradient: call it under torch.no_grad().
    """
    given = (x, weight, bias)
    if torch.is_grad_enabled() and any(t is not None and t.requires_grad for t in given):
        raise RuntimeError("layer_norm_int8 has no gradient: call it under torch.no_grad(), train through layer_norm")
    if getattr(forward_ad, "_current_level", 0) >= 0 and any(t is not None and forward_ad.unpack_dual(t).tangent is not None for t in given):
        raise RuntimeError("layer_norm_int8 has no gradient in forward mode either: give it primal tensors")
    _check(x, weight, bias)
    x2 = _rows(x, x.shape[-1])
    codes = torch.empty(x.shape, dtype=torch.int8, device=x.device)
    scales = torch.empty(x.shape[:-1], dtype=torch.float32, device=x.device)
    with torch.cuda.device(x.device):
        fq.fq_norm_forward(fq.FqNorm.from_torch(
            x2, y=codes.view(x2.shape), weight=None if weight is None else weight.contiguous(),
            bias=None if bias is None else bias.contiguous(), y_scale=scales.view(-1), eps=float(eps)))
    return codes, scales
