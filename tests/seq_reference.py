"""The operators of a selective state space block from their definitions, in
float64, with running bounds of the float32 arithmetic's rounding.

Every function returns, for each output, (value, bound): the bound is that of
a computation in float32 (unit roundoff U) from the same inputs whose
exponentials, reciprocals and square roots are within a few units.  It is
carried along with the values, term by term.  ``close`` adds the one rounding
to the output's type.

Tensors carry a mutant axis throughout ([mutants][tokens][channels]), of size
1 where shared; sequences are given by their lengths.
"""
import torch

U = 2.0 ** -24


def _sigmoid(z):
    """Value and relative bound: e^-z by an exponential of a rounded product
    (2 |z| U at the slope of at most 1), the sum, the quotient."""
    return 1 / (1 + torch.exp(-z)), (2 * z.abs().nan_to_num(0, 0, 0) + 10) * U


def _silu(z):
    s, rel = _sigmoid(z)
    return z * s, rel + U


def spans(lengths):
    row = 0
    for n in lengths:
        yield row, n
        row += n


def conv(x, taps, bias, lengths, activation=None, state=None):
    x, taps = x.double(), taps.double()
    M, (C, K), T, n = max(x.size(0), taps.size(0), 1 if bias is None else bias.size(0),
                          1 if state is None else state.size(0)), taps.shape[1:], x.size(1), len(lengths)
    bias = torch.zeros(1, C, dtype=torch.float64) if bias is None else bias.double()
    y, size = torch.zeros(M, T, C, dtype=torch.float64), torch.zeros(M, T, C, dtype=torch.float64)
    last = torch.zeros(M, n, K - 1, C, dtype=torch.float64)
    for i, (row, count) in enumerate(spans(lengths)):
        before = torch.zeros(M, K - 1, C, dtype=torch.float64) if state is None else state[:, i].double().expand(M, -1, -1)
        rows = torch.cat((before, x[:, row:row + count].expand(M, -1, -1)), 1)
        v, s = bias[:, None].expand(M, count, C).clone(), bias[:, None].abs().expand(M, count, C).clone()
        for k in range(K):
            v += taps[:, None, :, k] * rows[:, k:k + count]
            s += (taps[:, None, :, k] * rows[:, k:k + count]).abs()
        y[:, row:row + count], size[:, row:row + count] = v, s
        last[:, i] = rows[:, count:]
    bound = (K + 2) * U * size
    if activation == "silu":                    # its slope is at most 1.1
        y, rel = _silu(y)
        bound = 1.1 * bound + rel * y.abs()
    return (y, bound), (last, torch.zeros_like(last))


def softplus(s):
    """Value and relative bound: the exponential's argument is rounded once
    more (2 |s| U), logarithm, quotient and sums a few units."""
    return torch.logaddexp(s, torch.zeros_like(s)), (2 * s.abs().nan_to_num(0, 0, 0) + 14) * U


def scan(u, dt, A, B, C, lengths, skip=None, dt_bias=None, gate=None, use_softplus=True, state=None):
    given = [v for v in (u, dt, A, B, C, skip, dt_bias, gate, state) if v is not None]
    M = max(v.size(0) for v in given)
    D, N = A.shape[1:]
    T, n, G = u.size(1), len(lengths), B.size(-1) // N
    full = lambda v: v.double().expand(M, *v.shape[1:])  # noqa: E731
    u, dt, A, B, C = (full(v) for v in (u, dt, A, B, C))
    skip = torch.zeros(M, D, dtype=torch.float64) if skip is None else full(skip)
    dt_bias = torch.zeros(M, D, dtype=torch.float64) if dt_bias is None else full(dt_bias)
    y, by = torch.zeros(M, T, D, dtype=torch.float64), torch.zeros(M, T, D, dtype=torch.float64)
    out, bout = torch.zeros(M, n, D, N, dtype=torch.float64), torch.zeros(M, n, D, N, dtype=torch.float64)
    for i, (row, count) in enumerate(spans(lengths)):
        h = torch.zeros(M, D, N, dtype=torch.float64) if state is None else full(state)[:, i].clone()
        e = torch.zeros_like(h)                 # bound of h
        # a long sequence's decay over a chunk is one exponential of a sum of steps, at most 34 added in a row
        summed = (5 if count <= 512 else 40) * U
        for t in range(row, row + count):
            s = dt[:, t] + dt_bias
            step, rel = softplus(s) if use_softplus else (s, torch.zeros_like(s))
            rel = rel + U * s.abs().nan_to_num(0, 0, 0).clamp(min=1)         # the rounded sum: softplus' <= softplus
            b = B[:, t].view(M, G, 1, N).expand(M, G, D // G, N).reshape(M, D, N)
            c = C[:, t].view(M, G, 1, N).expand(M, G, D // G, N).reshape(M, D, N)
            x = step[..., None] * A
            a, into = torch.exp(x), (step * u[:, t])[..., None] * b
            # e^x: x within (rel + 3 U) of itself, the exponential 2 U; the products and the sum of the recurrence
            e = a * e + (a * h).abs() * (x.abs().nan_to_num(0, 0, 0) * (rel[..., None] + summed) + 4 * U) + into.abs() * (rel[..., None] + 5 * U)
            h = a * h + into
            v, size = (c * h).sum(-1), (c * h).abs().sum(-1)
            bound = (c.abs() * e).sum(-1) + (N + 6) * U * size + 3 * U * (skip * u[:, t]).abs()
            v = v + skip * u[:, t]
            bound = bound + U * v.abs()
            if gate is not None:
                g, grel = _silu(full(gate)[:, t])
                bound = bound * g.abs() + (v * g).abs() * (grel + U)
                v = v * g
            y[:, t], by[:, t] = v, bound
        out[:, i], bout[:, i] = h, e
    return (y, by), (out, bout)


def _norm(v, bound, kind, weight, bias, eps):
    """The norm of v, known within `bound`: each mean is a sum of `width` terms
    over lanes of at most 32 terms each and a tree or row of 32 more."""
    terms = 64 * U
    if kind == "layer":
        mean = v.mean(-1, keepdim=True)
        off = terms * v.abs().mean(-1, keepdim=True) + bound.mean(-1, keepdim=True)
        v, bound = v - mean, bound + off + U * (v.abs() + mean.abs())
    square = (v * v).mean(-1, keepdim=True) + eps
    f = square.rsqrt()
    # d f / f = - d square / (2 square)
    rel = (terms * square + 2 * (v.abs() * bound).mean(-1, keepdim=True) + (bound * bound).mean(-1, keepdim=True)) / (2 * square)
    out, bound = v * f, f * (bound + v.abs() * (rel + 4 * U))
    if weight is not None:
        w = weight.double()[:, None]
        out, bound = out * w, (bound + U * out.abs()) * w.abs()
    if bias is not None:
        out = out + bias.double()[:, None]
        bound = bound + U * (out.abs() + bias.double()[:, None].abs())
    return out, bound


def block_norm(y, residual=None, gate=None, gate_at="before", gate_activation="silu", after=None, after_weight=None, after_bias=None,
               scale=1.0, before=None, before_weight=None, before_bias=None, eps=1e-5):
    given = [v for v in (y, residual, gate, after_weight, after_bias, scale, before_weight, before_bias) if isinstance(v, torch.Tensor)]
    M = max(v.size(0) for v in given)
    v = y.double().expand(M, -1, -1)
    bound = torch.zeros_like(v)
    if gate is not None:
        z = gate.double()
        g, rel = {"silu": _silu, "sigmoid": _sigmoid, None: lambda z: (z, torch.zeros_like(z))}[gate_activation](z)
    if gate is not None and gate_at == "before":
        v = v * g
        bound = v.abs() * (rel + U)
    if after is not None:
        v, bound = _norm(v, bound, after, after_weight, after_bias, eps)
    if gate is not None and gate_at == "after":
        bound = bound * g.abs() + (v * g).abs() * (rel + U)
        v = v * g
    s = scale.double()[:, None] if isinstance(scale, torch.Tensor) else torch.tensor(float(torch.tensor(scale, dtype=torch.float32)), dtype=torch.float64)
    bound = bound * s.abs() + 2 * U * (v * s).abs()
    v = v * s
    if residual is not None:
        v = v + residual.double()
    bound = bound + U * v.abs()
    r = (v, bound)
    return r, None if before is None else _norm(v, bound, before, before_weight, before_bias, eps)


def close(got, expected, what=""):
    """got (float32 or bfloat16) is the expected value, within its bound and one
    rounding to got's type; infinities and NaN stand where they are expected."""
    value, bound = expected
    got = got.detach().cpu()
    assert got.shape == value.shape, f"{what}: shape {tuple(got.shape)}, not {tuple(value.shape)}"
    half = 2.0 ** -8 if got.dtype == torch.bfloat16 else U    # 8 and 24 significant bits
    tiny = 2.0 ** -126                          # results below it may be flushed
    g = got.double()
    finite = torch.isfinite(value)
    assert torch.equal(torch.isnan(g), torch.isnan(value)), f"{what}: NaN elsewhere"
    inf = torch.isinf(value)
    assert torch.equal(g[inf], value[inf]), f"{what}: infinities"
    off = (g - value).abs()[finite]
    most = (bound * (1 + half) + half * value.abs() + tiny)[finite]
    worst = float((off / most).max()) if off.numel() else 0.0
    assert worst <= 1.0, f"{what}: {worst:.3g} of the bound, {float(off.max()):.3g} off"
    return worst
