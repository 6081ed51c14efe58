"""B200-native truncated spectral layer (the single-GPU hot path of DTST).

`from paper_2607_14394_b200 import Plan` gives the ctypes binding of the C-ABI
library `libdtst.so`; `paper_2607_14394_b200.inputs` holds the seeded synthetic
input generators; `RmsNorm`, `GatedScan`, `Fp8Linear` (module `memory`) are the
operators of a recurrent memory around the layer, `LayerNorm`,
`CausalConv`, `SelectiveScan`, `GradNorm` (module `selective`) those of a selective one and its training step.  The binding is imported lazily so that the input generators
can be used without torch or the built library.
"""

_MEMORY = ("RmsNorm", "Fp8Linear", "GatedScan", "quantize_fp8", "quantize_fp8_weight", "FieldMemory", "RolloutMemory")
_SELECTIVE = ("LayerNorm", "CausalConv", "SelectiveScan", "GradNorm", "clip_grad_norm", "SelectiveMemory")
__all__ = ["Plan", "FNO", "binding", "inputs", "build", "memory", "selective", *_MEMORY, *_SELECTIVE]


def __getattr__(name):
    if name == "Plan":
        from .binding import Plan
        return Plan
    if name == "FNO":
        from .fno import FNO
        return FNO
    if name in _MEMORY:
        from . import memory
        return getattr(memory, name)
    if name in _SELECTIVE:
        from . import selective
        return getattr(selective, name)
    if name in ("binding", "inputs", "build", "memory", "selective"):
        import importlib
        return importlib.import_module("." + name, __name__)
    raise AttributeError(name)
