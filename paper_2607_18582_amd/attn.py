"""The operators of an attention block (``include/mure_attn.h``): ``rotate`` and
``attend`` of a ``Sequences`` (``Mure.sequences``), and ``Mure.gated``, which
works row by row.

Tensors, mutant axes, strides, streams and gradients are as in ``seq.py``: rows
of tokens, [tokens][heads * head_dim], or those of each mutant.
"""
from __future__ import annotations

import ctypes as C
from typing import Optional, Sequence

from .calls import call, native, one_of

ATTN_EXPORTED = ["mure_attn_version", "mure_attn_rotate", "mure_attn_attend", "mure_attn_gated"]
ATTN_VERSION = 1
ACTIVATIONS = {None: 0, "silu": 1, "sigmoid": 2, "relu": 3, "gelu": 4, "gelu_tanh": 5}
NORMS = {None: 0, "rms": 1, "layer": 2}


def declare(lib: C.CDLL) -> None:
    """Result and argument types of the calls of mure_attn.h."""
    P = C.c_void_p
    for name, res, args in (("mure_attn_version", C.c_int32, []), ("mure_attn_rotate", C.c_int, [P, P]),
                            ("mure_attn_attend", C.c_int, [P, P]), ("mure_attn_gated", C.c_int, [P, P])):
        f = getattr(lib, name)
        f.restype, f.argtypes = res, args


class AttnBatch:
    """The calls of mure_attn.h that a batch of sequences has."""

    def rotate(self, q, k, frequencies, *, head_dim: int, norm: Optional[str] = None, q_weight=None, k_weight=None,
               eps: float = 1e-6, positions=None, past=None, sections: Optional[Sequence[int]] = None,
               interleaved: bool = False, q_out=None, k_out=None):
        """Norm of every head's queries and keys, and rotation of their pairs of channels by
        position times frequency.

        q [tokens][heads * head_dim], k likewise or None; norm None, "rms" or "layer" over a
        head's channels, with weights [head_dim] float32; frequencies [pairs] float32, of
        channels (i, i + pairs) or, interleaved, (2 i, 2 i + 1).  A token's position is its
        place in its sequence plus past [sequences] int32; or positions [axes][tokens] int32,
        of which the first turns the first sections[0] pairs, and so on.  Returns (q_out,
        k_out), which may be q and k themselves."""
        if positions is not None and sections is None:
            sections = list(getattr(frequencies, "shape", ()))[-1:]
        return call(self.mure, self.args.rotate, self._open(), self.mure.device, self.count, self.tokens, q, k, frequencies,
                    head_dim, one_of(NORMS, norm, "norm"), q_weight, k_weight, eps, positions, past,
                    () if sections is None else tuple(sections), bool(interleaved), q_out, k_out)

    def attend(self, q, k, v, *, head_dim: int, scale: Optional[float] = None, causal: bool = True,
               window: Optional[int] = None, cache=None, past=None, out=None):
        """Attention of every token over its sequence.

        q [tokens][heads * head_dim]; k, v [tokens][kv_heads * head_dim]; a token sees the keys
        up to its own (causal) or all, less than `window` places away.  scale: 1 /
        sqrt(head_dim) without it.  cache: (keys, values), each [sequences][rows][kv_heads *
        head_dim], whose first past [sequences] int32 rows (none without it) come before the
        call's tokens; the call adds its own behind them.  Returns out, as q."""
        return call(self.mure, self.args.attend, self._open(), self.mure.device, self.count, self.tokens, q, k, v, head_dim, scale,
                    bool(causal), window, None if cache is None else tuple(cache), past, out)[0]


class AttnOps:
    """The calls of mure_attn.h that a context has."""

    def gated(self, x, gate, up, *, gate_bias=None, up_bias=None, activation: Optional[str] = "silu", out=None):
        """Gated feed-forward layer: activation(x gate^T + gate_bias) * (x up^T + up_bias).

        x [rows][inputs]; gate, up [outputs][inputs] in x's type; biases [outputs] float32;
        activation None, "silu", "sigmoid", "relu", "gelu" or "gelu_tanh".  Returns out
        [rows][outputs]."""
        if not self.ctx:
            raise ValueError("the context is closed")
        return call(self, native(self.lib).gated, self.ctx.value, self.device, x, gate, up, gate_bias, up_bias,
                    one_of(ACTIVATIONS, activation, "activation"), out)[0]
