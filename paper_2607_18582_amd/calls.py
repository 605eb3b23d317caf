"""What the calls on tensors share (``seq.py``, ``attn.py``): the native
marshalling module (``pyext/``), and a call's order with torch's streams."""
from __future__ import annotations

import ctypes as C

_args = _raw_stream = None                      # the native marshalling; torch's current stream of a device


def native(lib: C.CDLL):
    """The marshalling module, bound to the library; raises if it has not been built."""
    global _args, _raw_stream
    if _args is None:
        import torch
        try:
            from . import _seq_args
        except ImportError as e:
            raise RuntimeError("_seq_args.so is missing or stale: build it first "
                               "(python -m paper_2607_18582_amd.build)") from e
        for bind, calls in ((_seq_args.bind, (lib.mure_seq_conv, lib.mure_seq_scan, lib.mure_seq_norm)),
                            (_seq_args.bind_attn, (lib.mure_attn_rotate, lib.mure_attn_attend, lib.mure_attn_gated))):
            bind(*(C.cast(f, C.c_void_p).value for f in calls))
        _raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or \
            (lambda device: torch.cuda.current_stream(device).cuda_stream)
        _args = _seq_args
    return _args


def call(mure, fn, *args):
    """fn's two results, the call on the context's stream ordered with torch's current one."""
    device = mure.device
    if device < 0 or _raw_stream(device) == mure.stream:
        status, a, b = fn(*args)
    else:
        from torch import cuda
        current = cuda.current_stream(device)
        own = cuda.ExternalStream(mure.stream, device=device) if mure.stream else cuda.default_stream(device)
        own.wait_stream(current)
        status, a, b = fn(*args)
        current.wait_stream(own)
    if status:
        mure._check(status)
    return a, b


def one_of(table: dict, key, what: str) -> int:
    if key is None or isinstance(key, str):
        code = table.get(key)
        if code is not None:
            return code
    raise ValueError(f"{what} is {key!r}; one of {', '.join(map(repr, table))} is needed")
