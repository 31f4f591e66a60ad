"""MI355X-native MoR (Mixture of Representations) analyse-select-quantize path.

``binding``   ctypes front end of the C-ABI library ``libmor.so`` (HIP kernels for gfx950);
``mx``        the same for microscaled 4-bit operands, their products and tokens sorted by expert (``mor_mx.h``);
``mx_layers`` a linear layer and a layer of experts made of those, with their gradients, and an example of their use;
``build``     compiles that library in-tree with hipcc;
``workloads`` seeded synthetic BF16 operands (no method arithmetic).
"""
__all__ = ["binding", "build", "mx", "mx_layers", "workloads"]
