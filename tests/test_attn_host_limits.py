"""The operators of an attention block on the host, at their limits: calls of
as many mutants, heads and rows as they may have reach the device, and what is
not there is not read."""
import random

import pytest

from paper_2607_18582_amd import MURE_E_INVALID, MURE_E_UNSUPPORTED, Mure
from test_attn_host import CAP, D, G, Buffers, Cache, attend_args, call, put, rotate_args


@pytest.fixture()
def mure():
    m = Mure(device=-1)
    yield m
    m.close()


def apart(a, rows):
    """Caches of `rows` rows one behind the other, everything else behind them: nothing is read there."""
    width, n = a.kv_heads * a.head_dim, 3
    a.capacity = rows
    for c in (a.k_cache, a.v_cache):
        c.row_stride, c.seq_stride, c.mutant_stride = width, rows * width, 0
    for t in (a.k, a.v):
        t.mutant_stride = 0
    a.v_cache.p = a.k_cache.p + n * 2 * rows * width
    for i, name in enumerate(("q", "k", "v", "past", "out")):
        put(a, name if name == "past" else name + ".p", a.v_cache.p + (1 << 42) + i * (1 << 36))


@pytest.mark.parametrize("mutants,heads,kv_heads,dim,rows", [
    (128, 32, 8, 128, 131072), (32, 64, 64, 64, 262144), (65535, 4, 4, 8, 4096), (1, 1024, 1, 256, 1 << 30), (65535, 1024, 1024, 1, 1 << 20)])
@pytest.mark.parametrize("cache", [True, False])
def test_many_blocks(mure, mutants, heads, kv_heads, dim, rows, cache):
    a = attend_args(Buffers())
    a.n_mutants, a.heads, a.kv_heads, a.head_dim = mutants, heads, kv_heads, dim
    a.q.row_stride = a.out.row_stride = heads * dim
    a.q.mutant_stride = a.out.mutant_stride = 7 * heads * dim
    a.k.row_stride = a.v.row_stride = kv_heads * dim
    apart(a, rows)
    if not cache:
        a.k_cache.p = a.v_cache.p = a.past = None
    st, msg = call(mure, "attend", a)
    assert st == MURE_E_UNSUPPORTED and "planning-only" in msg, msg


def test_rows_of_a_cache(mure):
    a = attend_args(Buffers())
    for rows, status, word in ((1 << 30, MURE_E_UNSUPPORTED, "planning-only"), ((1 << 30) + 1, MURE_E_UNSUPPORTED, "too many rows"), (1 << 31, MURE_E_INVALID, "capacity")):
        apart(a, rows)
        st, msg = call(mure, "attend", a)
        assert st == status and word in msg, (rows, msg)


@pytest.mark.parametrize("p", [None, "keys"])
def test_a_weight_of_keys_that_are_not_there(mure, p):
    """Nothing checks such a weight's address, so nothing may read it."""
    a = rotate_args(Buffers())
    a.k_heads = 0
    a.k.p = a.k_out.p = None
    a.k_weight.p = 8 if p else None
    st, msg = call(mure, "rotate", a)
    if p:
        assert st == MURE_E_INVALID and "k_weight without" in msg, msg
    else:
        assert st == MURE_E_UNSUPPORTED and "planning-only" in msg, msg


W = G * D                                      # channels of a row of keys


@pytest.mark.parametrize("order", ["seq kv rows", "mutant kv seq rows", "kv mutant seq rows", "mutant seq kv rows", "seq mutant kv rows", "rows kv seq", "rows seq kv mutant"])
def test_caches_as_an_axis_of_one_tensor(mure, order):
    """Keys and values beside each other at any depth of one tensor; an element further they overlap."""
    a = attend_args(Buffers())
    base, stride, sizes = a.k_cache.p, {}, {"seq": 3, "rows": CAP, "mutant": 2, "kv": 2}
    at = W
    for axis in reversed(order.split()):
        stride[axis] = at
        at *= sizes[axis]
    if "mutant" not in stride:
        stride["mutant"] = 0
        a.k.mutant_stride = a.v.mutant_stride = 0
    a.k_cache = Cache(base, stride["mutant"], stride["seq"], stride["rows"])
    a.v_cache = Cache(base + 2 * stride["kv"], stride["mutant"], stride["seq"], stride["rows"])
    st, msg = call(mure, "attend", a)
    assert st == MURE_E_UNSUPPORTED and "planning-only" in msg, msg
    for off in (-1, 1):
        a.v_cache.p = base + 2 * (stride["kv"] + off)
        st, msg = call(mure, "attend", a)
        if off < 0 or order.split()[0] != "kv":            # behind everything there is room
            assert st == MURE_E_INVALID and "v_cache overlaps k_cache" in msg, (off, msg)


def test_accepted_caches_are_apart(mure):
    """Random layouts of both caches in one buffer: no call is accepted whose caches share an element."""
    rng, taken, refused = random.Random(7), 0, 0
    sizes = {"seq": 3, "rows": 4, "mutant": 2}
    buffers = Buffers()
    a = attend_args(buffers)
    base = buffers(1 << 20)
    a.capacity = sizes["rows"]
    for _ in range(4000):
        elements = []
        for c in (a.k_cache, a.v_cache):
            order, stride, at = rng.sample(list(sizes), 3), {}, W
            for axis in order:
                stride[axis] = at + rng.choice((0, 0, W, at, 3))
                at = stride[axis] * (sizes[axis] - 1) + at if rng.random() < 0.3 else stride[axis] * sizes[axis]
            start = rng.choice((0, W, 2 * W, rng.randrange(4 * W), rng.randrange(40 * W)))
            c.p, c.mutant_stride, c.seq_stride, c.row_stride = base + 2 * start, stride["mutant"], stride["seq"], stride["rows"]
            elements.append({start + m * stride["mutant"] + s * stride["seq"] + r * stride["rows"] + e
                             for m in range(2) for s in range(3) for r in range(4) for e in range(W)})
        st, msg = call(mure, "attend", a)
        if st == MURE_E_UNSUPPORTED:
            taken += 1
            assert not elements[0] & elements[1]
        elif "v_cache overlaps k_cache" in msg:
            refused += 1
    assert taken > 100 and refused > 100
