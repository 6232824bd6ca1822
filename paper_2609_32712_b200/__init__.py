"""B200-native MassAlloc Attention (MALA) hot path: C-ABI library ``libmala.so`` + thin binding.

``paper_2609_32712_b200.mala``      -- binding of the C ABI declared in ``include/mala.h`` (ctypes; ``_native.so`` for the calls that a decode step waits for)
``paper_2609_32712_b200.autograd``  -- ``mala_attention`` and its like: the forward / backward pairs as ``torch.autograd`` functions
``paper_2609_32712_b200.workloads`` -- seeded synthetic input generators (no method arithmetic)
"""
__version__ = "0.1.0"
