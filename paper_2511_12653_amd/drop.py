"""Torch front door to dropout: `dropout(x, p, seed, step, residual)`, one fq_dropout call forward and one backward.

The mask is a hash of place, seed and step: it is worked out again by the backward pass, and nothing is saved.  Marshalling only; torch owns
the memory and the stream (the current one).  There is no CPU path: CPU tensors raise.
"""
import torch
from torch.autograd.function import once_differentiable

from . import binding as fq


def _call(x, y, p, seed, step, residual):
    number, on_device = (0, step) if torch.is_tensor(step) else (step, None)
    with torch.cuda.device(x.device):
        fq.fq_dropout(fq.FqDropout.from_torch(x, y, p, seed, number, residual, on_device))


class _Dropout(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, residual, p, seed, step, out_dtype):
        if not x.is_cuda:
            raise RuntimeError("dropout runs on the GPU only (no CPU fallback)")
        if residual is not None and residual.shape != x.shape:
            raise ValueError("residual %s is not of x's shape %s" % (tuple(residual.shape), tuple(x.shape)))
        if residual is not None and out_dtype is not None and residual.dtype != out_dtype:
            raise TypeError("the result is of residual's type, %s" % residual.dtype)
        x = x.contiguous()
        y = torch.empty(x.shape, dtype=out_dtype or (x if residual is None else residual).dtype, device=x.device)
        _call(x, y, p, seed, step, None if residual is None else residual.contiguous())
        # (saved, so that a step that has been moved on before the backward pass is seen)
        ctx.save_for_backward(*((step,) if torch.is_tensor(step) else ()))
        ctx.meta = p, seed, step if not torch.is_tensor(step) else None, x.dtype
        return y

    @staticmethod
    @once_differentiable
    def backward(ctx, gy):
        p, seed, step, dtype = ctx.meta
        gx = None
        if ctx.needs_input_grad[0]:
            g = gy.contiguous()
            gx = torch.empty(g.shape, dtype=dtype, device=g.device)
            _call(g, gx, p, seed, ctx.saved_tensors[0] if step is None else step, None)
        return gx, (gy if ctx.needs_input_grad[1] else None), None, None, None, None


def dropout(x, p, seed, step=0, residual=None, out_dtype=None):
    """x / (1 - p) where a counter-based generator says so, else 0, plus residual.

    x: float16 or float32.  residual: a tensor of x's shape, float16 or float32, whose type the result then has; without one it is x's, or
    out_dtype.  seed, step: whole numbers of 64 bits; the same ones make the same mask for as many elements.  Give each layer a seed
    and each call of it a new step; step may be one int64 on the GPU, which a captured graph then moves on itself (after the
    backward pass).  Differentiable with respect to x and residual, once.
    """
    return _Dropout.apply(x, residual, float(p), int(seed), step if torch.is_tensor(step) else int(step), out_dtype)
