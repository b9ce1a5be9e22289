"""The compiled part of the Python bindings (csrc/binding.cpp): checks of tensors and the
library's calls for int8.py, rope.py and norm.py.  If it has not been built, every call
raises: there is no fallback."""
from __future__ import annotations

import ctypes
import os

from . import echo, fp8

ENTRIES = ("echo_int8_quantize", "echo_int8_gemm", "echo_rope_rotate", "echo_norm_join")

_module = None


def binding():
    global _module
    if _module is None:
        import torch
        path = os.path.join(os.path.dirname(os.path.abspath(__file__)), "_binding.so")
        if not os.path.exists(path):
            raise ImportError(f"{path} is missing: build it with "
                              "`python -c 'import __graft_entry__ as g; g.build()'`")
        from . import _binding
        L = echo.lib()
        gpu = torch.cuda.is_available()
        if gpu:
            torch.cuda.current_device()   # initialises
        _binding.setup(fp8.refuse, echo._check, torch._C._cuda_getDevice if gpu else None,
                       torch._C._cuda_getCurrentRawStream if gpu else None,
                       *[ctypes.cast(getattr(L, n), ctypes.c_void_p).value for n in ENTRIES])
        _module = _binding
    return _module
