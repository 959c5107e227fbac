"""Torch front door to the low-rank adapters: `add_adapters(base, x, ids, a, b)`, one fq_adapters_forward call.

Marshalling only; torch owns the memory (output and workspace come from its caching allocator) and the stream (the current one).  There is
no CPU path: CPU tensors raise.  There is no gradient either, as in `linear_int8`, beside which this serves: an adapter trains, by
itself, through float products.
"""
import torch
from torch.autograd import forward_ad

from . import binding as fq


def add_adapters(base, x, ids, a, b, scale=None, x_scale=None, out=None, out_dtype=None):
    """y = base + scale[id] * (x a[id]^T) b[id]^T for every token, with the adapter that `ids` names for it (or base itself).

    base: [..., n], float16 or float32: what the shared layer gave.  x: [..., k], float16, float32 or int8 codes with x_scale (float32, one
    per token or one for all): what it took.  ids: one integer per token; any outside [0, count) means no adapter.  a: [count, rank, k],
    b: [count, n, rank], float16, contiguous.  scale: count float32 values or None.  out: [..., n] float16 or float32, may be base
    itself; made in out_dtype (default: base's type) if not given.
    """
    given = (base, x, a, b, scale, x_scale, out)
    if torch.is_grad_enabled() and any(t is not None and t.requires_grad for t in given):
        raise RuntimeError("add_adapters has no gradient: call it under torch.no_grad()")
    if getattr(forward_ad, "_current_level", 0) >= 0 and any(t is not None and forward_ad.unpack_dual(t).tangent is not None for t in given):
        raise RuntimeError("add_adapters has no gradient in forward mode either: give it primal tensors")
    if not x.is_cuda:
        raise RuntimeError("add_adapters runs on the GPU only (no CPU fallback)")
    if x.dim() < 1 or a.dim() != 3 or b.dim() != 3 or x.shape[-1] != a.shape[2] or tuple(base.shape) != (*x.shape[:-1], b.shape[1]):
        raise ValueError("base %s, x %s, a %s and b %s do not fit" % tuple(tuple(t.shape) for t in (base, x, a, b)))
    if ids.dtype.is_floating_point or ids.dtype == torch.bool:
        raise TypeError("ids must be whole numbers")
    m, k, n = x.shape[:-1].numel(), x.shape[-1], b.shape[1]
    if ids.shape != x.shape[:-1] and ids.shape != (m,):
        raise ValueError("ids %s are not one for each of x's %s tokens" % (tuple(ids.shape), tuple(x.shape[:-1])))
    if ids.dtype != torch.int32:               # (an int64 that is none of the adapters must not become one)
        ids = ids.long().clamp(-1, a.shape[0]).to(torch.int32)
    if out is None:
        out, own = torch.empty(base.shape, dtype=out_dtype or base.dtype, device=x.device), True
    else:
        if out.shape != base.shape or (out_dtype is not None and out.dtype != out_dtype):
            raise ValueError("out must have shape %s and the wanted type" % (tuple(base.shape),))
        own = False

    def rows(t, width):
        t = t.reshape(m, width)
        return t.contiguous() if (width > 1 and t.stride(1) != 1) or (m > 1 and t.stride(0) < width) else t

    with torch.cuda.device(x.device):
        y = out.view(m, n)                     # (raises where the rows are no view of it)
        d = fq.FqAdapters.from_torch(rows(x, k), ids.reshape(-1).contiguous(), a, b, y, base=y if out is base else rows(base, n), scale=scale,
                                     x_scale=None if x_scale is None else x_scale.reshape(-1).contiguous())
        workspace = torch.empty(fq.fq_adapters_workspace_bytes(d), dtype=torch.uint8, device=x.device)
        fq.fq_adapters_forward(d, workspace)
    if not own and not out.is_inference():
        torch.autograd.graph.increment_version(out)       # (a backward pass that has saved it is told)
    return out
