"""The operators of an attention block from their definitions, in float64, with
bounds of the float32 arithmetic's rounding, as in ``seq_reference``: every
function returns (value, bound) for each output, and ``seq_reference.close``
adds the one rounding to the output's type.

Tensors carry a mutant axis throughout ([mutants][tokens][channels]), of size
1 where shared; sequences are given by their lengths.
"""
import math

import torch

from seq_reference import U, _norm, _sigmoid, close, spans  # noqa: F401

HALF = {torch.float32: 0.0, torch.bfloat16: 2.0 ** -8}   # the weights' own rounding: none, and half a step of 8 bits


def rotate(x, frequencies, lengths, head_dim, norm=None, weight=None, eps=1e-6, past=None, positions=None, sections=None,
           interleaved=False):
    """One of q and k.  Angles are exact products; cosine and sine come from a remainder rounded once (|r| <= pi/4: U) and
    series of at most six terms of decreasing size (3 U): 4 U each."""
    M = max(x.size(0), frequencies.size(0), 1 if weight is None else weight.size(0))
    T, pairs = x.size(1), frequencies.size(-1)
    at = torch.zeros(T, dtype=torch.float64)
    for i, (row, n) in enumerate(spans(lengths)):
        at[row:row + n] = torch.arange(n) + (0 if past is None else int(past[i]))
    at = at[:, None].expand(T, pairs)
    if positions is not None:
        at = torch.cat([p[:, None].expand(T, c) for p, c in zip(positions.double(), sections)], 1)
    angle = at * frequencies.double()[:, None]               # [M or 1][T][pairs]
    cos, sin = torch.cos(angle)[:, :, None], torch.sin(angle)[:, :, None]
    v = x.double().expand(M, -1, -1).unflatten(-1, (-1, head_dim))
    bound = torch.zeros_like(v)
    if norm:
        flat, fb = _norm(v.flatten(1, 2), bound.flatten(1, 2), norm, None if weight is None else weight.expand(M, -1), None, eps)
        v, bound = flat.view_as(v), fb.view_as(v)
    v, bound = v.clone(), bound.clone()
    if pairs:
        first, second = (slice(0, 2 * pairs, 2), slice(1, 2 * pairs, 2)) if interleaved else (slice(0, pairs), slice(pairs, 2 * pairs))
        a, b, ea, eb = v[..., first].clone(), v[..., second].clone(), bound[..., first].clone(), bound[..., second].clone()
        off = 4 * U * (a.abs() + b.abs())
        v[..., first], v[..., second] = a * cos - b * sin, a * sin + b * cos
        bound[..., first] = ea * cos.abs() + eb * sin.abs() + off + 3 * U * ((a * cos).abs() + (b * sin).abs())
        bound[..., second] = ea * sin.abs() + eb * cos.abs() + off + 3 * U * ((a * sin).abs() + (b * cos).abs())
    return v.flatten(-2), bound.flatten(-2)


def attend(q, k, v, lengths, head_dim, scale=None, causal=True, window=None, cache=None, past=None):
    """Returns (out, bound) and the caches afterwards.

    A weight's exponent: a sum of head_dim products, scaled, less the largest so far: its absolute error is that of the sum
    and of a few roundings of numbers as large as the largest exponent.  The weights' sums add their roundings (at most one a
    key), a rescaling a tile of at least 32 keys two more, and the join of parts three.  In bfloat16 every weight is rounded once before it meets
    its value."""
    M = max(t.size(0) for t in (q, k, v) + tuple(cache or ()))
    dtype, H, G = q.dtype, q.size(-1) // head_dim, k.size(-1) // head_dim
    scale = float(torch.tensor(head_dim ** -0.5 if scale is None else scale, dtype=torch.float32))
    qd, kd, vd = (t.double().expand(M, -1, -1) for t in (q, k, v))
    held = None if cache is None else [c.clone() for c in cache]
    out, err = (torch.full((M, q.size(1), H * head_dim), float("nan"), dtype=torch.float64) for _ in range(2))
    for i, (row, n) in enumerate(spans(lengths)):
        p = 0 if past is None else int(past[i])
        if n == 0:
            continue
        if cache is not None and (p < 0 or p + n > cache[0].size(-2)):
            err[:, row:row + n] = 0
            continue
        keys, vals = kd[:, row:row + n], vd[:, row:row + n]
        if cache is not None:
            for c, new in zip(held, (k, v)):
                c[:, i, p:p + n] = new[:c.size(0), row:row + n]
            keys, vals = (torch.cat((c[:, i, :p].double().expand(M, -1, -1), t), 1) for c, t in zip(cache, (keys, vals)))
        at, j = torch.arange(p, p + n)[:, None], torch.arange(p + n)
        seen = torch.ones(n, p + n, dtype=torch.bool)
        if causal:
            seen &= j <= at
        if window:
            seen &= (j - at).abs() < window
        for h in range(H):
            g = slice(h // (H // G) * head_dim, (h // (H // G) + 1) * head_dim)
            qh, kh, vh = qd[:, row:row + n, h * head_dim:(h + 1) * head_dim], keys[..., g], vals[..., g]
            s = (qh[:, :, None] * kh[:, None]).sum(-1) * scale
            size = (qh[:, :, None] * kh[:, None]).abs().sum(-1) * abs(scale)
            s = s.masked_fill(~seen, float("-inf"))
            top = s.amax(-1, keepdim=True)
            w = torch.exp(s - top)
            w = torch.where(seen, w, torch.zeros((), dtype=torch.float64))
            w = w / w.sum(-1, keepdim=True)
            steps = (p + n + 2 * ((p + n) // 32 + 2) + 8) * U
            largest = s.abs().masked_fill(~seen, 0).amax(-1, keepdim=True)
            eps = (head_dim + 4) * U * size.masked_fill(~seen, 0) + 8 * U * (largest + 1)
            # a key that is hidden counts for nothing, whatever its value is
            wv = w[..., None] * vh[:, None]
            wv = torch.where(seen[None, :, :, None], wv, torch.zeros((), dtype=torch.float64))
            o = wv.sum(2)
            e = (wv.abs() * (eps + HALF[dtype] + steps)[..., None]).sum(2) + o.abs() * ((w * eps).sum(-1, keepdim=True) + steps)
            out[:, row:row + n, h * head_dim:(h + 1) * head_dim] = o
            err[:, row:row + n, h * head_dim:(h + 1) * head_dim] = 1.01 * e
    return (out, err), held


def activation(a, bound, kind):
    """Value and bound: the slopes are at most 1.13; erf and the hyperbolic tangent are good to a few units of 1."""
    if kind is None:
        return a, bound
    if kind == "relu":
        return a.clamp(min=0), bound
    if kind == "sigmoid":
        s, rel = _sigmoid(a)
        return s, 0.25 * bound + rel * s
    if kind == "silu":
        s, rel = _sigmoid(a)
        return a * s, 1.13 * bound + (rel + U) * (a * s).abs()
    if kind == "gelu":
        y = 0.5 * a * (1 + torch.erf(a * 0.5 ** 0.5))
        return y, 1.13 * bound + 8 * U * a.abs() + 3 * U * y.abs()
    u = math.sqrt(2 / math.pi) * (a + 0.044715 * a ** 3)
    y = 0.5 * a * (1 + torch.tanh(u))
    s, rel = _sigmoid(2 * u)                                 # y = a sigmoid(2 u); u is rounded a few times
    return y, 1.13 * bound + (rel + 16 * u.abs() * U + 2 * U) * y.abs()


def gated(x, gate, up, gate_bias=None, up_bias=None, kind="silu"):
    given = [t for t in (x, gate, up, gate_bias, up_bias) if t is not None]
    M, K = max(t.size(0) for t in given), x.size(-1)

    def project(w, b):
        xs, ws = x.double().expand(M, -1, -1), w.double().expand(M, -1, -1).transpose(1, 2).contiguous()
        v, size = torch.bmm(xs, ws), torch.bmm(xs.abs(), ws.abs())
        if b is not None:
            v, size = v + b.double()[:, None], size + b.double().abs()[:, None]
        return v, (K + 2) * U * size

    a, ea = project(gate, gate_bias)
    b, eb = project(up, up_bias)
    a, ea = activation(a, ea, kind)
    return a * b, a.abs() * eb + b.abs() * ea + ea * eb + U * (a * b).abs()
