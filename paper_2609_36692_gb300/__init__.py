"""GB300 (sm_103a) implementation of the NormPre optimizer step.

The product is ``libnormpre.so`` (C ABI declared in ``include/normpre.h``);
``normpre`` is its ctypes binding; ``optim`` (the optimizer step) and ``layers``
(packed attention and 8-bit activation checkpoints, which produce the step's
gradients) only marshal torch tensors into those calls.
"""
from . import normpre  # noqa: F401
