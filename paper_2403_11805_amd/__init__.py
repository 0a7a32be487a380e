"""Chunk-wise KV-cache scoring, compression and swap-in for LLM context
switching (arXiv 2403.11805) on one MI355X: a C-ABI library of hand-written
gfx950 kernels (csrc/, built into libkvswitch.so) and this thin binding.

`synth` (seeded inputs) imports nothing from the binding; the binding is loaded
on first attribute access so that importing the package never needs the library.
"""
from __future__ import annotations

import importlib
import sys

__all__ = ["binding", "build", "synth"]

_BINDING = f"{__name__}.binding"


def __getattr__(name):
    if name in __all__:
        return importlib.import_module(f"{__name__}.{name}")
    # looked up in the binding every time, so that what is replaced there is replaced here too (0.4 us; import_module takes 3)
    binding = sys.modules.get(_BINDING) or importlib.import_module(_BINDING)
    try:
        return getattr(binding, name)
    except AttributeError:
        raise AttributeError(f"module {__name__!r} has no attribute {name!r}") from None
