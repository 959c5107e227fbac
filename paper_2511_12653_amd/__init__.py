"""Fused learnable-scale fake quantization for MI355X (gfx950).

`workloads` generates seeded synthetic inputs (numpy only).  The GPU entry points live in
`binding` (thin ctypes marshalling onto the C-ABI library built from csrc/); it is imported
on first use and raises if the compiled library is missing -- there is no CPU fallback.
`fake_quantize` (module `autograd`) wraps the forward and backward calls in a torch.autograd Function, `linear_int8` (module
`linear`) the int8 linear layer, `AdamW` (module `optim`) the multi-tensor AdamW step in a torch.optim.Optimizer.
"""
from . import workloads  # noqa: F401

_API = ("fq_forward", "fq_backward", "fq_multi_tensor", "fq_workspace_bytes", "fq_workspace_init",
        "fq_validate", "fq_status_string", "fq_plan_create", "fq_plan_run", "fq_plan_run_adam", "fq_plan_destroy",
        "fq_layout", "FqLayoutInfo", "fq_distill_loss", "fq_distill_workspace_bytes", "FqDistill", "FqTensor", "FqAdam", "FqTensorArray", "fq_tensor_array", "FqError", "library_path",
        "fq_linear_forward", "fq_linear_workspace_bytes", "FqLinear", "fq_adamw_create", "fq_adamw_step", "fq_adamw_destroy",
        "fq_adamw_workspace_bytes", "FqParam", "FqAdamW", "FQ_I8", "FQ_STATE_F32", "FQ_STATE_F8",
        "FQ_F16", "FQ_F32", "FQ_FLAG_NO_DX", "FQ_FLAG_TWO_PASS", "FQ_FLAG_NO_POLL", "FQ_MODE_FORWARD", "FQ_MODE_BACKWARD")


_FRONT_DOORS = {"fake_quantize": "autograd", "linear_int8": "linear", "AdamW": "optim"}


def __getattr__(name):
    if name in _FRONT_DOORS:
        import importlib
        return getattr(importlib.import_module(__name__ + "." + _FRONT_DOORS[name]), name)
    if name == "binding" or name in _API:
        import importlib
        mod = importlib.import_module(__name__ + ".binding")
        return mod if name == "binding" else getattr(mod, name)
    raise AttributeError(name)
