"""Torch front door to the int8 linear layer: `linear_int8(x, w, w_scale, ...)`, one fq_linear_forward call.

Marshalling only; torch owns the memory (output and workspace come from its caching allocator) and the stream (the current
one).  There is no CPU path: CPU tensors raise.  There is no gradient either: codes are constants, and a network trains
through `fake_quantize` and the float product, whose values these are.
"""
import torch
from torch.autograd import forward_ad

from . import binding as fq


def linear_int8(x, w, w_scale, bias=None, x_scale=None, out=None, out_dtype=None):
    """y = x_scale * w_scale * (codes of x) (codes of w)^T + bias.

    x: [..., k], float16 or float32 (quantized row by row: scale = largest magnitude / 127) or int8 codes with x_scale
    (float32, one per row or one for all).  w: [n, k] int8 codes, w_scale: float32, n values or one, both as `fq_forward`
    writes them.  bias: n float32 values or None.  out: [..., n] float16 or float32, made in out_dtype (default: x's type, or
    float16 for codes) if not given.
    """
    if torch.is_grad_enabled() and any(t is not None and t.requires_grad for t in (x, w_scale, bias, x_scale, out)):
        raise RuntimeError("linear_int8 has no gradient: call it under torch.no_grad(), train through fake_quantize")
    # (outside every forward-mode level, which a torch that counts them says, there is no tangent: 0.1 us instead of 0.9)
    if getattr(forward_ad, "_current_level", 0) >= 0 and any(
            t is not None and forward_ad.unpack_dual(t).tangent is not None for t in (x, w_scale, bias, x_scale, out)):
        raise RuntimeError("linear_int8 has no gradient in forward mode either: give it primal tensors")
    if not x.is_cuda:
        raise RuntimeError("linear_int8 runs on the GPU only (no CPU fallback)")
    if x.dim() < 1 or w.dim() != 2 or x.shape[-1] != w.shape[1]:
        raise ValueError("x %s and w %s do not fit" % (tuple(x.shape), tuple(w.shape)))
    n, k = w.shape
    rows = x.numel() // k if k else x.shape[:-1].numel()
    shape = (*x.shape[:-1], n)
    given = out
    if out is None:
        out = torch.empty(shape, dtype=out_dtype or (torch.float16 if x.dtype == torch.int8 else x.dtype), device=x.device)
        y = out.view(rows, n)
    else:
        if tuple(out.shape) != shape or (out_dtype is not None and out.dtype != out_dtype):
            raise ValueError("out must have shape %s and the wanted type" % (shape,))
        y = out.view(rows, n)                       # (raises where the rows are no view of it)
    x2 = x.reshape(rows, k)
    if (k > 1 and x2.stride(1) != 1) or (rows > 1 and x2.stride(0) < k):
        x2 = x2.contiguous()                        # (values apart, or an expanded x whose rows are the same memory)
    with torch.cuda.device(x.device):
        d = fq.FqLinear.from_torch(x2, w, w_scale, y, bias=bias, x_scale=x_scale)
        workspace = torch.empty(fq.fq_linear_workspace_bytes(d), dtype=torch.uint8, device=x.device)
        fq.fq_linear_forward(d, workspace)
    if given is not None and not given.is_inference():
        torch.autograd.graph.increment_version(given)      # (a backward pass that has saved it is told)
    return out
