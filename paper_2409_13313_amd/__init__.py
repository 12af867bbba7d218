"""FP64 GEMM emulated on the gfx950 INT8 matrix cores (Ozaki scheme, ozIMMU_H form).

`ozimmu` and `mx` (the bindings to the C-ABI HIP library: emulated FP64 products, microscaled 4-bit
operators) are imported lazily so that the input generators can be used on machines without the built library.
"""

__all__ = ["inputs", "mx", "ozimmu"]


def __getattr__(name):
    if name in ("ozimmu", "mx", "inputs"):
        import importlib
        return importlib.import_module(f"{__name__}.{name}")
    raise AttributeError(name)
