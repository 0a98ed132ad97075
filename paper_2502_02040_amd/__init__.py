"""MI355X (gfx950) implementation of the M2R2 dual-stream decode path.

The compute runs in ``libm2r2.so`` (hand-written HIP kernels behind the C ABI
declared in ``include/m2r2.h``); ``binding`` marshals arguments to it, and
``kv8`` to the operators of the 8-bit paged cache (``include/m2r2_kv8.h``).
"""
from .binding import (Model, PagedKV, M2R2Error, lib, workspace_size, EXPORTS)  # noqa: F401
from .kv8 import KV8Pages, kv8_append, kv8_attention, kv8_workspace  # noqa: F401

__all__ = ["Model", "PagedKV", "M2R2Error", "lib", "workspace_size", "EXPORTS", "KV8Pages", "kv8_append",
           "kv8_attention", "kv8_workspace"]
