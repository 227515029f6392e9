"""MI355X (gfx950) sparse parameter store: pull rows by key, compute per-task
gradients, push them back merged per key with an AdaGrad update.

The computation lives in the HIP library ``libadapm_hip.so`` (C ABI in
``include/adapm.h``); ``Store`` and ``dedup`` only marshal torch tensors into
it.  Importing this package loads nothing; the library is loaded on first use
and a missing library is an error, never a fallback.
"""
import importlib

_STORE = ("Store", "StagedStore", "dedup", "action_timing")
_OPERATORS = ("ClipPlan", "MX4", "clip_grads", "grad_norm", "mx4_product", "mx4_quantize")

__all__ = [*_STORE, *_OPERATORS, "workloads"]


def __getattr__(name):
    if name in _STORE:
        module = "store"
    elif name in _OPERATORS:
        module = "operators"
    elif name == "workloads":
        return importlib.import_module(__name__ + ".workloads")
    else:
        raise AttributeError(name)
    value = getattr(importlib.import_module(__name__ + "." + module), name)
    globals()[name] = value   # found without this function from now on
    return value
