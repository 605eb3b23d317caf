"""The operators of a selective state space block (``include/mure_seq.h``):
``Mure.sequences`` registers the lengths of a test set's sequences and returns
a ``Sequences``, whose ``conv`` and ``scan`` run over them (and the operators of
``attn.py``); ``Mure.block_norm`` works row by row.

Argument marshalling only, as in ``binding.py``, the tensors' part of it in C++
(``pyext/seq_args.cpp``).  Activations are CUDA tensors of packed rows,
``[tokens][channels]`` where all mutants share them or
``[mutants][tokens][channels]``; parameters and states likewise have a leading
mutant axis or none.  A size-1 or expanded (stride 0) mutant axis counts as
shared.  Rows may be strided (slices of a projection's output); a row's
channels are contiguous.  Results have a mutant axis when any argument has.
There are no gradients: a tensor that requires one is refused outside
``torch.no_grad()``, and so is one with a forward tangent.

The library enqueues on its context's stream.  Where another stream is
current in torch, the call is ordered after that stream's work and that stream
after the call.
"""
from __future__ import annotations

import ctypes as C
from typing import Optional, Sequence

import numpy as np

from .attn import AttnBatch
from .calls import call as _call, native as _native, one_of as _one_of

SEQ_EXPORTED = ["mure_seq_version", "mure_seq_create", "mure_seq_destroy", "mure_seq_conv", "mure_seq_scan",
                "mure_seq_norm"]
SEQ_VERSION = 1
ACTIVATIONS = {None: 0, "silu": 1, "sigmoid": 2}
NORMS = {None: 0, "rms": 1, "layer": 2}
GATES = {"before": 1, "after": 2}


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


class Sequences(AttnBatch):
    """A batch of sequences of ``lengths`` tokens, packed one after the other.
    Made by ``Mure.sequences``.  It has to outlive the graphs that captured its
    calls; each of them keeps a workspace of its own here."""

    def __init__(self, mure, lengths: Sequence[int]):
        self.mure, self.handle, self.args = mure, C.c_void_p(), _native(mure.lib)
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

    def _open(self) -> int:
        if not self.handle:
            raise ValueError("the batch is closed")
        return self.handle.value

    def conv(self, x, taps, bias=None, *, activation: Optional[str] = None, state=None, state_out=None, out=None):
        """Causal depthwise convolution along every sequence.

        x [tokens][channels]; taps [channels][K] in x's type; bias [channels] float32;
        activation None or "silu"; state [sequences][K - 1][channels], the rows before the
        first token (zeros without it).  Returns (out, state_out), state_out being the last
        K - 1 rows of (state, x); both may be given, state_out as the state itself."""
        return _call(self.mure, self.args.conv, self._open(), self.mure.device, self.count, self.tokens, x, taps, bias,
                     _one_of(ACTIVATIONS, activation, "activation"), state, state_out, out)

    def scan(self, u, dt, A, B, C_, *, skip=None, dt_bias=None, gate=None, softplus: bool = True, state=None,
             state_out=None, out=None):
        """Selective scan along every sequence.

        u, dt, gate [tokens][channels]; A [channels][states] float32; B, C_
        [tokens][groups * states] in u's type; skip, dt_bias [channels] float32; state
        [sequences][channels][states] float32 (zeros without it).  Returns (out,
        state_out); both may be given, state_out as the state itself."""
        return _call(self.mure, self.args.scan, self._open(), self.mure.device, self.count, self.tokens, u, dt, A, B, C_,
                     skip, dt_bias, gate, bool(softplus), state, state_out, out)


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
        if not self.ctx:
            raise ValueError("the context is closed")
        return _call(self, _native(self.lib).norm, self.ctx.value, self.device, y, residual, gate,
                     _one_of(GATES, gate_at, "gate_at"), _one_of(ACTIVATIONS, gate_activation, "gate_activation"),
                     _one_of(NORMS, after, "after"), after_weight, after_bias, scale, _one_of(NORMS, before, "before"),
                     before_weight, before_bias, eps, residual_out, out)
