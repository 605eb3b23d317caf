"""The operators at sizes whose work takes more than one round, run or launch,
and at offsets near and past 32 bits: the same bits as from small calls, which
``test_gpu_seq.py`` compares with the definitions."""
import pytest
import torch

from paper_2607_18582_amd import Mure

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def mure():
    m = Mure(device=0)
    yield m
    m.close()


@pytest.fixture(autouse=True)
def memory():
    yield
    torch.cuda.empty_cache()


def source(seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return lambda *s, dtype=torch.float32: torch.randn(*s, generator=g, device="cuda").to(dtype)


def rows_of(lengths):
    at = 0
    for n in lengths:
        yield slice(at, at + n)
        at += n


# ---------------------------------------------------------------- norms: more rows than blocks

@pytest.mark.parametrize("dtype,residual", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32")])
@pytest.mark.parametrize("width,M,rows", [(3, 700, 40), (60, 700, 40), (128, 700, 20), (250, 500, 11), (500, 500, 11), (1000, 400, 7),
                                          (2000, 400, 7), (4001, 100, 7), (8192, 100, 7), (16384, 60, 9)])
def test_norm_of_many_rows(mure, dtype, residual, width, M, rows):
    """Blocks go from row to row; a mutant alone has a block for each."""
    print(f"[large norm] {dtype}/{residual} {M} x {rows} x {width}", flush=True)
    r = source(width)
    y, z = r(M, rows, width, dtype=TYPES[dtype]), r(rows, width, dtype=TYPES[dtype])
    res = r(M, rows, width, dtype=TYPES[residual])
    aw, s, bw, bb = r(width), r(M, width), r(width), r(M, width)
    for options in (dict(after="layer", after_weight=aw, scale=s, before="rms", before_weight=bw, gate=z),
                    dict(before="layer", before_weight=bw, before_bias=bb),
                    dict(after="rms", gate=z, gate_at="after", gate_activation="sigmoid")):
        one = lambda m: {k: v[m] if v is s or v is bb else v for k, v in options.items()}  # noqa: E731
        got = mure.block_norm(y, res, **options)
        for m in (0, 1, M // 2, M - 1):
            expected = mure.block_norm(y[m], res[m], **one(m))
            for a, e in zip(got, expected):
                assert (a is None and e is None) or torch.equal(a[m], e), m
        if got[1] is not None:                  # in place: a row is read ahead of the stores of the row before it
            ys, rs = y.clone(), res.clone()
            mure.block_norm(ys, rs, residual_out=rs, out=ys, **options)
            assert torch.equal(rs, got[0]) and torch.equal(ys, got[1])


# ---------------------------------------------------------------- convolutions: long runs, many sequences, several launches

@pytest.mark.parametrize("dtype,C", [("f32", 1024), ("bf16", 2051)])
@pytest.mark.parametrize("K", [2, 4, 8])
def test_conv_in_long_runs(mure, dtype, C, K):
    print(f"[large conv] {dtype} C={C} K={K}", flush=True)
    lengths, M = [2000, 0, 33, 34, 1, 66, 2200, 5, 32], 4
    r, T = source(K), sum(lengths)
    x, taps, bias = r(T, C, dtype=TYPES[dtype]), r(M, C, K, dtype=TYPES[dtype]), r(C)
    state = r(M, len(lengths), K - 1, C, dtype=TYPES[dtype])
    held = state.clone()
    y, last = mure.sequences(lengths).conv(x, taps, bias, activation="silu", state=held, state_out=held)
    for m in (0, 3):
        for i, cut in enumerate(rows_of(lengths)):
            one, end = mure.sequences([lengths[i]]).conv(x[cut], taps[m], bias, activation="silu", state=state[m, i:i + 1])
            assert torch.equal(y[m, cut], one) and torch.equal(last[m, i:i + 1], end), (m, i)


@pytest.mark.parametrize("count", [40000, (1 << 17) + 5])
def test_many_short_sequences(mure, count):
    """Batches for which fewer kinds of runs are kept, against their halves."""
    print(f"[large] {count} sequences", flush=True)
    g = torch.Generator().manual_seed(count)
    lengths = torch.randint(0, 7, (count,), generator=g)
    r, T, C, N = source(1), int(lengths.sum()), 12, 4
    x, taps, state = r(T, C), r(C, 4), r(count, 3, C)
    A, b, c, h = -r(C, N).abs(), r(T, N), r(T, N), r(count, C, N)
    whole = mure.sequences(lengths.tolist())
    y, last = whole.conv(x, taps, activation="silu", state=state)
    ys, ends = whole.scan(x, x, A, b, c, state=h)
    half = count // 2
    row = int(lengths[:half].sum())
    for s, cut in ((slice(0, half), slice(0, row)), (slice(half, count), slice(row, T))):
        part = mure.sequences(lengths[s].tolist())
        a, e = part.conv(x[cut], taps, activation="silu", state=state[s])
        assert torch.equal(a, y[cut]) and torch.equal(e, last[s])
        a, e = part.scan(x[cut], x[cut], A, b[cut], c[cut], state=h[s])
        assert torch.equal(a, ys[cut]) and torch.equal(e, ends[s])


def test_conv_in_several_launches(mure):
    """2^20 channels: a launch holds 8192 runs.  Row t of x is the source from its element t on."""
    print("[large conv] launches", flush=True)
    T, C = 8200, 1 << 20
    base = source(2)(T + C, dtype=torch.bfloat16)
    taps = torch.ones(C, 1, dtype=torch.bfloat16, device="cuda")
    y, _ = mure.sequences([1] * T).conv(base.as_strided((T, C), (1, 1)), taps)
    for t in (0, 1, 8190, 8191, 8192, 8193, T - 1):
        assert torch.equal(y[t], base[t:t + C]), t


# ---------------------------------------------------------------- scans: several launches, many chunked sequences

@pytest.mark.parametrize("length", [1, 6])
def test_scan_in_several_launches(mure, length):
    """65535 mutants: a launch holds 256 sequences."""
    print(f"[large scan] launches of {length}", flush=True)
    r, M, n = source(3), 65535, 300
    u, dt, b, c = r(n * length, 1), r(n * length, 1), r(n * length, 1), r(n * length, 1)
    A, skip = -r(M, 1, 1).abs(), r(M, 1)
    seqs = mure.sequences([length] * n)
    y, last = seqs.scan(u, dt, A, b, c, skip=skip)
    for m in (slice(0, 40), slice(30000, 30040), slice(M - 40, M)):
        a, e = seqs.scan(u, dt, A[m], b, c, skip=skip[m])
        assert torch.equal(a, y[m]) and torch.equal(e, last[m])


def test_scan_of_many_chunked_sequences(mure):
    """More than 65535 sequences of more than one run, against smaller batches."""
    print("[large scan] chunked sequences", flush=True)
    count, length = 65600, 513
    r, T = source(4), 65600 * 513
    u, dt, b, c = r(T, 1), r(T, 1) - 3, r(T, 1), r(T, 1)
    A, state = -torch.ones(1, 1, device="cuda"), r(count, 1, 1)
    y, last = mure.sequences([length] * count).scan(u, dt, A, b, c, state=state)
    half = 40000
    for s in (slice(0, half), slice(half, count)):
        cut = slice(s.start * length, s.stop * length)
        a, e = mure.sequences([length] * (s.stop - s.start)).scan(u[cut], dt[cut], A, b[cut], c[cut], state=state[s])
        assert torch.equal(a, y[cut]) and torch.equal(e, last[s])


# ---------------------------------------------------------------- offsets

@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_scan_of_rows_nearly_too_far_apart(mure, dtype):
    """Four rows span just less than 2^32 bytes: the last distance that a lane keeps in 32 bits."""
    print(f"[large scan] far rows {dtype}", flush=True)
    r, T, D, N = source(5), 9, 70, 16
    far = ((1 << 32) // TYPES[dtype].itemsize - 1 - 64) // 3
    rows = torch.empty((T - 1) * far + D, dtype=TYPES[dtype], device="cuda").as_strided((T, D), (far, 1))
    u, dt, gate = (r(T, D, dtype=TYPES[dtype]) for _ in range(3))
    A, b, c = -r(D, N).abs(), r(T, N, dtype=TYPES[dtype]), r(T, N, dtype=TYPES[dtype])
    seqs = mure.sequences([T])
    expected, last = seqs.scan(u, dt, A, b, c, gate=gate)
    for name, near in (("u", u), ("dt", dt), ("gate", gate)):
        rows.copy_(near)
        given = dict({"u": u, "dt": dt, "gate": gate}, **{name: rows})
        y, state = seqs.scan(given["u"], given["dt"], A, b, c, gate=given["gate"])
        assert torch.equal(y, expected) and torch.equal(state, last), name
    y, state = seqs.scan(u, dt, A, b, c, gate=gate, out=rows)
    assert torch.equal(rows, expected) and torch.equal(state, last)


def test_mutants_far_apart(mure):
    """Mutants more than 2^32 bytes and 2^31 elements from each other, read and written."""
    print("[large] far mutants", flush=True)
    r, lengths, C, N, K = source(6), [600, 3], 24, 16, 4
    T, far = sum(lengths), (1 << 31) + 40
    dtype = torch.bfloat16
    memory = torch.empty(far + 4 * T * C, dtype=dtype, device="cuda")
    into = torch.empty(far + 4 * T * C, dtype=dtype, device="cuda")
    spread = lambda m, *s: m.as_strided((2, *s), (far, *torch.empty(s, device="meta").stride()))  # noqa: E731
    x, taps, bias, st = r(2, T, C, dtype=dtype), r(C, K, dtype=dtype), r(C), r(2, 2, K - 1, C, dtype=dtype)
    seqs = mure.sequences(lengths)
    y, last = seqs.conv(x, taps, bias, activation="silu", state=st)
    a, e = seqs.conv(spread(memory, T, C).copy_(x), taps, bias, activation="silu", state=st, out=spread(into, T, C))
    assert torch.equal(a, y) and torch.equal(e, last)
    a, e = seqs.conv(x, taps, bias, activation="silu", state=spread(memory, 2, K - 1, C).copy_(st), state_out=spread(into, 2, K - 1, C))
    assert torch.equal(a, y) and torch.equal(e, last)
    A, b, c, h = -r(C, N).abs(), r(T, N, dtype=dtype), r(T, N, dtype=dtype), r(2, 2, C, N)
    dt = r(2, T, C, dtype=dtype)
    y, last = seqs.scan(x, dt, A, b, c, state=h)
    a, e = seqs.scan(spread(memory, T, C).copy_(x), dt, A, b, c, state=h, out=spread(into, T, C))
    assert torch.equal(a, y) and torch.equal(e, last)
    a, e = seqs.scan(x, spread(memory, T, C).copy_(dt), A, b, c, state=h)
    assert torch.equal(a, y) and torch.equal(e, last)
    y, o = mure.block_norm(x, before="rms")
    a, e = mure.block_norm(spread(memory, T, C).copy_(x), before="rms", out=spread(into, T, C))
    assert torch.equal(a, y) and torch.equal(e, o)
