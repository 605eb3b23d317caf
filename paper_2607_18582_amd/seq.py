"""The operators of a selective state space block (``include/mure_seq.h``):
``Mure.sequences`` registers the lengths of a test set's sequences and returns
a ``Sequences``, whose ``conv`` and ``scan`` run over them; ``Mure.block_norm``
works row by row.

Argument marshalling only, as in ``binding.py``.  Activations are CUDA tensors
of packed rows, ``[tokens][channels]`` where all mutants share them or
``[mutants][tokens][channels]``; parameters and states likewise have a leading
mutant axis or none.  A size-1 or expanded (stride 0) mutant axis counts as
shared.  Rows may be strided (slices of a projection's output); a row's
channels are contiguous.  Results have a mutant axis when any argument has.

The library enqueues on its context's stream.  Where another stream is
current in torch, the call is ordered after that stream's work and that stream
after the call.
"""
from __future__ import annotations

import ctypes as C
from typing import Optional, Sequence

import numpy as np

SEQ_EXPORTED = ["mure_seq_version", "mure_seq_create", "mure_seq_destroy", "mure_seq_conv", "mure_seq_scan",
                "mure_seq_norm"]
SEQ_VERSION = 1
ACTIVATIONS = {None: 0, "silu": 1, "sigmoid": 2}
NORMS = {None: 0, "rms": 1, "layer": 2}
GATES = {"before": 1, "after": 2}


class _rows(C.Structure):                       # mure_seq_in, mure_seq_out
    _fields_ = [("p", C.c_void_p), ("mutant_stride", C.c_int64), ("row_stride", C.c_int64)]


class _param(C.Structure):                      # mure_seq_param
    _fields_ = [("p", C.c_void_p), ("mutant_stride", C.c_int64)]


class mure_seq_conv_args(C.Structure):
    _fields_ = [("dtype", C.c_int32), ("n_mutants", C.c_int32), ("channels", C.c_int32), ("n_taps", C.c_int32),
                ("activation", C.c_int32), ("reserved", C.c_int32), ("x", _rows), ("taps", C.c_void_p),
                ("taps_mutant_stride", C.c_int64), ("bias", _param), ("state", C.c_void_p),
                ("state_mutant_stride", C.c_int64), ("state_out", C.c_void_p),
                ("state_out_mutant_stride", C.c_int64), ("out", _rows)]


class mure_seq_scan_args(C.Structure):
    _fields_ = [("dtype", C.c_int32), ("n_mutants", C.c_int32), ("channels", C.c_int32), ("states", C.c_int32),
                ("groups", C.c_int32), ("softplus", C.c_int32), ("u", _rows), ("dt", _rows), ("b", _rows),
                ("c", _rows), ("gate", _rows), ("a", _param), ("skip", _param), ("dt_bias", _param),
                ("state", C.c_void_p), ("state_mutant_stride", C.c_int64), ("state_out", C.c_void_p),
                ("state_out_mutant_stride", C.c_int64), ("out", _rows)]


class mure_seq_norm_args(C.Structure):
    _fields_ = [("dtype", C.c_int32), ("residual_dtype", C.c_int32), ("n_mutants", C.c_int32),
                ("channels", C.c_int32), ("rows", C.c_int64), ("gate_at", C.c_int32), ("gate_activation", C.c_int32),
                ("after", C.c_int32), ("before", C.c_int32), ("eps", C.c_float), ("scale_all", C.c_float),
                ("y", _rows), ("gate", _rows), ("residual", _rows), ("after_weight", _param), ("after_bias", _param),
                ("scale", _param), ("before_weight", _param), ("before_bias", _param), ("residual_out", _rows),
                ("out", _rows)]


def declare(lib: C.CDLL) -> None:
    """Result and argument types of the calls of mure_seq.h."""
    P = C.c_void_p
    for name, res, args in (("mure_seq_version", C.c_int32, []),
                            ("mure_seq_create", C.c_int, [P, C.c_int64, P, C.POINTER(P)]),
                            ("mure_seq_destroy", None, [P]),
                            ("mure_seq_conv", C.c_int, [P, C.POINTER(mure_seq_conv_args)]),
                            ("mure_seq_scan", C.c_int, [P, C.POINTER(mure_seq_scan_args)]),
                            ("mure_seq_norm", C.c_int, [P, C.POINTER(mure_seq_norm_args)])):
        f = getattr(lib, name)
        f.restype, f.argtypes = res, args


class _Call:
    """The tensors of one call: their checks, the number of mutants, and the
    order against torch's current stream."""

    def __init__(self, mure, first, what: str):
        import torch
        self.torch, self.mure = torch, mure
        if not isinstance(first, torch.Tensor):
            raise TypeError(f"{what} must be a torch tensor")
        self.device, self.dtype = first.device, first.dtype
        if mure.device >= 0 and (self.device.type != "cuda" or self.device.index != mure.device):
            raise ValueError(f"{what} is on {self.device}, the context on cuda:{mure.device}")
        if self.dtype not in (torch.float32, torch.bfloat16):
            raise TypeError(f"{what} is {self.dtype}; float32 or bfloat16 is needed")
        if first.dim() not in (2, 3) or first.size(-1) >= 1 << 31:
            raise ValueError(f"{what} has shape {tuple(first.shape)}; [rows][channels] is needed, or that of each mutant")
        self.code = 0 if self.dtype is torch.float32 else 1
        self.mutants, self.axis = 1, False

    def _seen(self, t, what: str, dtype, shape, dense: bool):
        """The mutant stride of t, a tensor of `shape` or [mutants] + shape; dense:
        but for the mutant axis it is contiguous, else its last axis is."""
        if not isinstance(t, self.torch.Tensor):
            raise TypeError(f"{what} must be a torch tensor")
        if t.device != self.device or t.dtype is not dtype:
            raise TypeError(f"{what} is {t.dtype} on {t.device}; {dtype} on {self.device} is needed")
        have, extra = t.shape, t.dim() - len(shape)
        if not 0 <= extra <= 1 or have[extra:] != shape:
            raise ValueError(f"{what} has shape {tuple(have)}; {tuple(shape)} is needed, or that of each mutant")
        if dense:
            one = t[0] if extra and have[0] else t
            if not one.is_contiguous():
                raise ValueError(f"{what} must be contiguous" + (" for each mutant" if extra else ""))
        elif shape[-1] > 1 and t.stride(-1) != 1:
            raise ValueError(f"the last axis of {what} must be contiguous")
        if not extra:
            return 0
        self.axis = True
        n = have[0]
        if n == 0:
            raise ValueError(f"{what} has no mutants")
        if n == 1:
            return 0
        if self.mutants not in (1, n):
            raise ValueError(f"{what} has {n} mutants, another argument {self.mutants}")
        self.mutants = n
        return t.stride(0)

    def rows(self, t, what: str, rows: int, width: int, dtype=None):
        if t is None:
            return _rows()
        stride = self._seen(t, what, dtype or self.dtype, (rows, width), False)
        return _rows(t.data_ptr(), stride, t.stride(-2))

    def dense(self, t, what: str, shape, dtype=None):
        """(address, mutant stride)"""
        if t is None:
            return None, 0
        stride = self._seen(t, what, dtype or self.torch.float32, shape, True)
        return t.data_ptr(), stride

    def output(self, t, what: str, shape, dtype=None):
        """t, checked, or a new tensor of the call's mutants; and its strides."""
        full = (self.mutants, *shape) if self.axis else tuple(shape)
        if t is None:
            return self.torch.empty(full, dtype=dtype or self.dtype, device=self.device)
        if tuple(t.shape) != full or t.dtype is not (dtype or self.dtype) or t.device != self.device:
            raise ValueError(f"{what} is {tuple(t.shape)} {t.dtype}; {full} {dtype or self.dtype} is needed")
        if full[-1] > 1 and t.stride(-1) != 1:
            raise ValueError(f"the last axis of {what} must be contiguous")
        return t

    def out_rows(self, t):
        return _rows(t.data_ptr(), t.stride(0) if self.axis else 0, t.stride(-2))

    def out_dense(self, t, what: str):
        if not (t[0] if self.axis else t).is_contiguous():
            raise ValueError(f"{what} must be contiguous" + (" for each mutant" if self.axis else ""))
        return t.data_ptr(), t.stride(0) if self.axis else 0

    def run(self, fn, handle, args) -> None:
        mure = self.mure
        if mure.device < 0:
            mure._check(fn(handle, C.byref(args)))
            return
        current = self.torch.cuda.current_stream(self.device)
        if current.cuda_stream == mure.stream:
            mure._check(fn(handle, C.byref(args)))
            return
        own = self.torch.cuda.ExternalStream(mure.stream, device=self.device) if mure.stream else \
            self.torch.cuda.default_stream(self.device)
        own.wait_stream(current)
        try:
            mure._check(fn(handle, C.byref(args)))
        finally:
            current.wait_stream(own)


def _one_of(table: dict, key, what: str) -> int:
    try:
        return table[key]
    except (KeyError, TypeError):
        raise ValueError(f"{what} is {key!r}; one of {', '.join(map(repr, table))} is needed") from None


class Sequences:
    """A batch of sequences of ``lengths`` tokens, packed one after the other.
    Made by ``Mure.sequences``."""

    def __init__(self, mure, lengths: Sequence[int]):
        self.mure, self.handle = mure, C.c_void_p()
        given = np.asarray(lengths)
        if given.ndim != 1 or (given.size and given.dtype.kind not in "iu"):
            raise ValueError("lengths must be a list of whole numbers")
        self.lengths = given.astype(np.int64)
        self.lengths.setflags(write=False)
        mure._check(mure.lib.mure_seq_create(mure.ctx, self.lengths.size, C.c_void_p(self.lengths.ctypes.data),
                                             C.byref(self.handle)))
        self.count, self.tokens = self.lengths.size, int(self.lengths.sum())

    def close(self):
        if getattr(self, "handle", None):
            self.mure.lib.mure_seq_destroy(self.handle)
            self.handle = None

    __del__ = close

    def _call(self, first, what: str) -> _Call:
        if not self.handle:
            raise ValueError("the batch is closed")
        return _Call(self.mure, first, what)

    def conv(self, x, taps, bias=None, *, activation: Optional[str] = None, state=None, state_out=None, out=None):
        """Causal depthwise convolution along every sequence.

        x [tokens][channels]; taps [channels][K] in x's type; bias [channels] float32;
        activation None or "silu"; state [sequences][K - 1][channels], the rows before the
        first token (zeros without it).  Returns (out, state_out), state_out being the last
        K - 1 rows of (state, x); both may be given, state_out as the state itself."""
        c = self._call(x, "x")
        width, K = x.size(-1), taps.size(-1)
        a = mure_seq_conv_args(dtype=c.code, channels=width, n_taps=K,
                               activation=_one_of(ACTIVATIONS, activation, "activation"))
        held = (self.count, K - 1, width)
        a.x = c.rows(x, "x", self.tokens, width)
        a.taps, a.taps_mutant_stride = c.dense(taps, "taps", (width, K), c.dtype)
        a.bias = _param(*c.dense(bias, "bias", (width,)))
        a.state, a.state_mutant_stride = c.dense(state, "state", held, c.dtype)
        out = c.output(out, "out", (self.tokens, width))
        state_out = c.output(state_out, "state_out", held)
        a.state_out, a.state_out_mutant_stride = c.out_dense(state_out, "state_out")
        a.out, a.n_mutants = c.out_rows(out), c.mutants
        c.run(self.mure.lib.mure_seq_conv, self.handle, a)
        return out, state_out

    def scan(self, u, dt, A, B, C_, *, skip=None, dt_bias=None, gate=None, softplus: bool = True, state=None,
             state_out=None, out=None):
        """Selective scan along every sequence.

        u, dt, gate [tokens][channels]; A [channels][states] float32; B, C_
        [tokens][groups * states] in u's type; skip, dt_bias [channels] float32; state
        [sequences][channels][states] float32 (zeros without it).  Returns (out,
        state_out); both may be given, state_out as the state itself."""
        c = self._call(u, "u")
        width, N = u.size(-1), A.size(-1)
        cols = B.size(-1)
        if N == 0 or cols % N:
            raise ValueError(f"B has {cols} columns, no multiple of the {N} states of A")
        a = mure_seq_scan_args(dtype=c.code, channels=width, states=N, groups=cols // N, softplus=bool(softplus))
        T, held, f32 = self.tokens, (self.count, width, N), c.torch.float32
        a.u = c.rows(u, "u", T, width)
        a.dt = c.rows(dt, "dt", T, width)
        a.b = c.rows(B, "B", T, cols)
        a.c = c.rows(C_, "C_", T, cols)
        a.gate = c.rows(gate, "gate", T, width)
        a.a = _param(*c.dense(A, "A", (width, N)))
        a.skip = _param(*c.dense(skip, "skip", (width,)))
        a.dt_bias = _param(*c.dense(dt_bias, "dt_bias", (width,)))
        a.state, a.state_mutant_stride = c.dense(state, "state", held)
        out = c.output(out, "out", (T, width))
        state_out = c.output(state_out, "state_out", held, f32)
        a.state_out, a.state_out_mutant_stride = c.out_dense(state_out, "state_out")
        a.out, a.n_mutants = c.out_rows(out), c.mutants
        c.run(self.mure.lib.mure_seq_scan, self.handle, a)
        return out, state_out


class SeqOps:
    """The calls of mure_seq.h that a context has."""

    def sequences(self, lengths: Sequence[int]) -> Sequences:
        """Register a batch of sequences by their lengths (tokens, 0 or more each)."""
        s = Sequences(self, lengths)
        self._batches.add(s)
        return s

    def _close_batches(self):
        for s in list(getattr(self, "_batches", ())):
            s.close()

    def block_norm(self, y, residual=None, *, gate=None, gate_at: str = "before", gate_activation: Optional[str] = "silu",
                   after: Optional[str] = None, after_weight=None, after_bias=None, scale=1.0,
                   before: Optional[str] = None, before_weight=None, before_bias=None, eps: float = 1e-5,
                   residual_out=None, out=None):
        """The norms after a block and before the next, around the residual sum:
        r = residual + scale * after(y), gated by ``gate`` before or after that norm
        (gate_at), and before(r).  Norms: None, "rms" or "layer".

        y, gate [rows][channels]; residual the same, or float32; weights, biases and scale
        float32 [channels] (scale may be a number).  Returns (r, before(r)), the second None
        without ``before``; residual_out = False leaves r out (None); residual_out may be the
        residual and out may be y or the gate."""
        c = _Call(self, y, "y")
        rows, width = y.size(-2), y.size(-1)
        torch = c.torch
        rtype = c.dtype if residual is None else residual.dtype
        a = mure_seq_norm_args(dtype=c.code, residual_dtype=0 if rtype is torch.float32 else 1, channels=width, rows=rows,
                               gate_at=0 if gate is None else _one_of(GATES, gate_at, "gate_at"),
                               gate_activation=_one_of(ACTIVATIONS, gate_activation, "gate_activation"),
                               after=_one_of(NORMS, after, "after"), before=_one_of(NORMS, before, "before"),
                               eps=eps, scale_all=1.0 if isinstance(scale, torch.Tensor) else scale)
        if rtype not in (torch.float32, torch.bfloat16):
            raise TypeError(f"residual is {rtype}; float32 or bfloat16 is needed")
        a.y = c.rows(y, "y", rows, width)
        a.gate = c.rows(gate, "gate", rows, width)
        a.residual = c.rows(residual, "residual", rows, width, rtype)
        for name, t in (("after_weight", after_weight), ("after_bias", after_bias),
                        ("scale", scale if isinstance(scale, torch.Tensor) else None),
                        ("before_weight", before_weight), ("before_bias", before_bias)):
            if t is not None:
                setattr(a, name, _param(*c.dense(t, name, (width,))))
        a.n_mutants = c.mutants
        if residual_out is not False:
            residual_out = c.output(residual_out, "residual_out", (rows, width), rtype)
            a.residual_out = c.out_rows(residual_out)
        else:
            residual_out = None
        if before is not None:
            out = c.output(out, "out", (rows, width))
            a.out = c.out_rows(out)
        elif out is not None:
            raise ValueError("out needs a `before` norm")
        c.run(self.lib.mure_seq_norm, self.ctx, a)
        return residual_out, out
