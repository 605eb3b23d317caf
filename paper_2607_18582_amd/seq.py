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
import struct
import sys
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
                            ("mure_seq_conv", C.c_int, [P, P]), ("mure_seq_scan", C.c_int, [P, P]),
                            ("mure_seq_norm", C.c_int, [P, P])):
        f = getattr(lib, name)
        f.restype, f.argtypes = res, args


# The argument blocks as they are filled here: one pack is several times as fast as a Structure's fields, and
# a call on single tokens takes no longer on the GPU than its marshalling.
_CONV = struct.Struct("=6i14q")
_SCAN = struct.Struct("=6i28q")
_NORM = struct.Struct("=4iq4i2f25q")
assert (_CONV.size, _SCAN.size, _NORM.size) == tuple(map(C.sizeof, (mure_seq_conv_args, mure_seq_scan_args, mure_seq_norm_args)))

_NONE_ROWS, _NONE = (0, 0, 0), (0, 0)


class _Call:
    """The tensors of one call: their checks, the number of mutants, and the
    order against torch's current stream."""

    __slots__ = ("mure", "torch", "device", "dtype", "code", "mutants", "axis", "first")

    def __init__(self, mure, first, what: str):
        torch = self.torch = sys.modules["torch"]
        if not isinstance(first, torch.Tensor):
            raise TypeError(f"{what} must be a torch tensor")
        self.mure, self.first, self.dtype, self.device = mure, first, first.dtype, first.get_device()
        if self.device != mure.device:                 # -1: the CPU, or a planning-only context
            raise ValueError(f"{what} is on {first.device}, the context on device {mure.device}")
        if self.dtype is torch.bfloat16:
            self.code = 1
        elif self.dtype is torch.float32:
            self.code = 0
        else:
            raise TypeError(f"{what} is {self.dtype}; float32 or bfloat16 is needed")
        if not 2 <= first.dim() <= 3 or first.shape[-1] >= 1 << 31:
            raise ValueError(f"{what} has shape {tuple(first.shape)}; [rows][channels] is needed, or that of each mutant")
        self.mutants, self.axis = 1, False

    def _check(self, t, what: str, dtype):
        if not isinstance(t, self.torch.Tensor):
            raise TypeError(f"{what} must be a torch tensor")
        if t.dtype is not dtype or t.get_device() != self.device:
            raise TypeError(f"{what} is {t.dtype} on {t.device}; {dtype} on {self.first.device} is needed")

    def _mutant_axis(self, n: int, stride: int, what: str) -> int:
        """The mutant stride of an axis of n mutants."""
        self.axis = True
        if n == 1:
            return 0
        if n == 0 or self.mutants not in (1, n):
            raise ValueError(f"{what} has {n} mutants, another argument {self.mutants}")
        self.mutants = n
        return stride

    def rows(self, t, what: str, rows: int, width: int, dtype=None):
        """(address, mutant stride, row stride) of [rows][width] or that of each mutant"""
        if t is None:
            return _NONE_ROWS
        self._check(t, what, dtype or self.dtype)
        shape, stride = t.shape, t.stride()
        if shape[-2:] != (rows, width) or len(shape) > 3:
            raise ValueError(f"{what} has shape {tuple(shape)}; {(rows, width)} is needed, or that of each mutant")
        if stride[-1] != 1 and width > 1:
            raise ValueError(f"the last axis of {what} must be contiguous")
        if len(shape) == 2:
            return t.data_ptr(), 0, stride[0]
        return t.data_ptr(), self._mutant_axis(shape[0], stride[0], what), stride[1]

    def dense(self, t, what: str, shape: tuple, dtype=None):
        """(address, mutant stride) of a tensor of `shape`, contiguous, or that of each mutant"""
        if t is None:
            return _NONE
        self._check(t, what, dtype or self.torch.float32)
        have, extra = t.shape, t.dim() - len(shape)
        if not 0 <= extra <= 1 or have[extra:] != shape:
            raise ValueError(f"{what} has shape {tuple(have)}; {shape} is needed, or that of each mutant")
        if not t.is_contiguous() and not (extra and have[0] and t[0].is_contiguous()):
            raise ValueError(f"{what} must be contiguous" + (" for each mutant" if extra else ""))
        return t.data_ptr(), self._mutant_axis(have[0], t.stride(0), what) if extra else 0

    def output(self, t, what: str, shape: tuple, dtype=None):
        """t, checked, or a new tensor of the call's mutants."""
        full = (self.mutants, *shape) if self.axis else shape
        if t is None:
            return self.first.new_empty(full, dtype=dtype or self.dtype)
        self._check(t, what, dtype or self.dtype)
        if t.shape != full:
            raise ValueError(f"{what} has shape {tuple(t.shape)}; {full} is needed")
        return t

    def out_rows(self, t, what: str):
        stride = t.stride()
        if stride[-1] != 1 and t.shape[-1] > 1:
            raise ValueError(f"the last axis of {what} must be contiguous")
        return t.data_ptr(), stride[0] if self.axis else 0, stride[-2]

    def out_dense(self, t, what: str):
        if not t.is_contiguous() and not (self.axis and t[0].is_contiguous()):
            raise ValueError(f"{what} must be contiguous" + (" for each mutant" if self.axis else ""))
        return t.data_ptr(), t.stride(0) if self.axis else 0

    def run(self, fn, handle, args: bytes) -> None:
        mure, cuda = self.mure, self.torch.cuda
        if mure.device < 0 or cuda.current_stream(self.device).cuda_stream == mure.stream:
            status = fn(handle, args)
        else:
            current = cuda.current_stream(self.device)
            own = cuda.ExternalStream(mure.stream, device=self.device) if mure.stream else cuda.default_stream(self.device)
            own.wait_stream(current)
            status = fn(handle, args)
            current.wait_stream(own)
        if status:
            mure._check(status)


def _one_of(table: dict, key, what: str) -> int:
    if key is None or isinstance(key, str):
        code = table.get(key)
        if code is not None:
            return code
    raise ValueError(f"{what} is {key!r}; one of {', '.join(map(repr, table))} is needed")


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
        width, K = x.shape[-1], taps.shape[-1]
        held = (self.count, K - 1, width)
        px, ptaps = c.rows(x, "x", self.tokens, width), c.dense(taps, "taps", (width, K), c.dtype)
        pbias, pstate = c.dense(bias, "bias", (width,)), c.dense(state, "state", held, c.dtype)
        out, state_out = c.output(out, "out", (self.tokens, width)), c.output(state_out, "state_out", held)
        c.run(self.mure.lib.mure_seq_conv, self.handle,
              _CONV.pack(c.code, c.mutants, width, K, _one_of(ACTIVATIONS, activation, "activation"), 0, *px, *ptaps, *pbias,
                         *pstate, *c.out_dense(state_out, "state_out"), *c.out_rows(out, "out")))
        return out, state_out

    def scan(self, u, dt, A, B, C_, *, skip=None, dt_bias=None, gate=None, softplus: bool = True, state=None,
             state_out=None, out=None):
        """Selective scan along every sequence.

        u, dt, gate [tokens][channels]; A [channels][states] float32; B, C_
        [tokens][groups * states] in u's type; skip, dt_bias [channels] float32; state
        [sequences][channels][states] float32 (zeros without it).  Returns (out,
        state_out); both may be given, state_out as the state itself."""
        c = self._call(u, "u")
        width, N, cols, T = u.shape[-1], A.shape[-1], B.shape[-1], self.tokens
        if N == 0 or cols % N:
            raise ValueError(f"B has {cols} columns, no multiple of the {N} states of A")
        held = (self.count, width, N)
        pu, pdt, pb, pc = c.rows(u, "u", T, width), c.rows(dt, "dt", T, width), c.rows(B, "B", T, cols), c.rows(C_, "C_", T, cols)
        pz, pa = c.rows(gate, "gate", T, width), c.dense(A, "A", (width, N))
        pskip, pbias = c.dense(skip, "skip", (width,)), c.dense(dt_bias, "dt_bias", (width,))
        pstate = c.dense(state, "state", held)
        out = c.output(out, "out", (T, width))
        state_out = c.output(state_out, "state_out", held, c.torch.float32)
        c.run(self.mure.lib.mure_seq_scan, self.handle,
              _SCAN.pack(c.code, c.mutants, width, N, cols // N, bool(softplus), *pu, *pdt, *pb, *pc, *pz, *pa, *pskip, *pbias,
                         *pstate, *c.out_dense(state_out, "state_out"), *c.out_rows(out, "out")))
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
        torch, (rows, width) = c.torch, y.shape[-2:]
        rtype = c.dtype if residual is None else residual.dtype
        if rtype is not c.dtype and rtype is not torch.float32:
            raise TypeError(f"residual is {rtype}; {c.dtype} or float32 is needed")
        if before is None and out is not None:
            raise ValueError("out needs a `before` norm")
        py, pz = c.rows(y, "y", rows, width), c.rows(gate, "gate", rows, width)
        pr, w = c.rows(residual, "residual", rows, width, rtype), (width,)
        scaled = isinstance(scale, torch.Tensor)
        params = (*c.dense(after_weight, "after_weight", w), *c.dense(after_bias, "after_bias", w),
                  *c.dense(scale if scaled else None, "scale", w), *c.dense(before_weight, "before_weight", w),
                  *c.dense(before_bias, "before_bias", w))
        pro = po = _NONE_ROWS
        if residual_out is False:
            residual_out = None
        else:
            residual_out = c.output(residual_out, "residual_out", (rows, width), rtype)
            pro = c.out_rows(residual_out, "residual_out")
        if before is not None:
            out = c.output(out, "out", (rows, width))
            po = c.out_rows(out, "out")
        c.run(self.lib.mure_seq_norm, self.ctx,
              _NORM.pack(c.code, 0 if rtype is torch.float32 else 1, c.mutants, width, rows,
                         0 if gate is None else _one_of(GATES, gate_at, "gate_at"),
                         _one_of(ACTIVATIONS, gate_activation, "gate_activation"), _one_of(NORMS, after, "after"),
                         _one_of(NORMS, before, "before"), eps, 1.0 if scaled else scale, *py, *pz, *pr, *params, *pro, *po))
        return residual_out, out
