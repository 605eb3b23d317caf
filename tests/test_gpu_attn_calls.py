"""How the operators of an attention block are called: together, captured into
graphs, on other streams, over long caches, in and out of batches, with strides
and alignments of every kind."""
import ctypes as C

import pytest
import torch

import attn_reference as R
from paper_2607_18582_amd import Mure, MureError
from test_gpu_attn import TYPES, cuda, normal, qkv, say

pytestmark = pytest.mark.gpu

MIXED = [40, 1, 700, 16, 0, 130, 17, 65, 3, 128]       # every class of lengths, in each type


@pytest.fixture(scope="module")
def mure():
    m = Mure(device=0)
    yield m
    m.close()


@pytest.fixture()
def own():
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        m = Mure(device=0)
    yield m, side
    torch.cuda.synchronize()
    m.close()


def starts(lengths):
    return [sum(lengths[:i]) for i in range(len(lengths))]


def caches(seed, n, capacity, width, dtype, M=1):
    g = torch.Generator().manual_seed(seed)
    return tuple(normal(g, M, n, capacity, width, dtype=dtype) for _ in range(2))


# ---------------------------------------------------------------- in and out of batches

@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("window", [None, 50])
def test_a_sequence_alone_and_in_a_batch(mure, dtype, window):
    say(f"[alone] {dtype} window={window}")
    dim, M = 64, 3
    q, k, v = cuda(*qkv(1, MIXED, 4, 2, dim, TYPES[dtype], M))
    past = torch.tensor([5, 2200, 0, 600, 4, 1500, 1030, 0, 511, 1023], dtype=torch.int32).cuda()
    held = cuda(*caches(2, len(MIXED), 2600, 2 * dim, TYPES[dtype], M))
    f = torch.rand(32).cuda()
    seqs = mure.sequences(MIXED)
    whole = seqs.attend(q, k, v, head_dim=dim, window=window)
    turned, _ = seqs.rotate(q, None, f, head_dim=dim, norm="rms", past=past)
    after = [c.clone() for c in held]
    over = seqs.attend(q, k, v, head_dim=dim, window=window, cache=after, past=past)
    for i, (s, n) in enumerate(zip(starts(MIXED), MIXED)):
        one = mure.sequences([n])
        for m in (0, 2):
            at = (m, slice(s, s + n))
            assert torch.equal(one.attend(q[at], k[at], v[at], head_dim=dim, window=window), whole[at]), (i, m)
            alone = [c[m, i:i + 1].clone() for c in held]
            p = past[i:i + 1]
            assert torch.equal(one.attend(q[at], k[at], v[at], head_dim=dim, window=window, cache=alone, past=p), over[at]), (i, m)
            for c, a, new in zip(alone, after, (k, v)):
                assert torch.equal(c[0], a[m, i])
                assert torch.equal(c[0, int(p):int(p) + n], new[at])
            assert torch.equal(one.rotate(q[at], None, f, head_dim=dim, norm="rms", past=p)[0], turned[at]), (i, m)
    # a cache with more rows behind it
    more = [torch.cat((c, torch.full_like(c, float("nan"))), 2) for c in held]
    assert torch.equal(seqs.attend(q, k, v, head_dim=dim, window=window, cache=more, past=past), over)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("dim", [64, 40, 128, 98, 250, 34])
def test_strides_and_alignment(mure, dtype, dim):
    """Rows that are no aligned pieces of 16 bytes, spread over wider ones, mutants inside tokens: the same bits."""
    say(f"[strides] {dtype} dim={dim}")
    H, G, M, dt = 4, 2, 2, TYPES[dtype]
    q, k, v = cuda(*qkv(3, MIXED, H, G, dim, dt, M))
    past = torch.tensor([5, 700, 0, 600, 4, 300, 100, 0, 511, 10], dtype=torch.int32).cuda()
    held = cuda(*caches(4, len(MIXED), 720, G * dim, dt, M))
    seqs = mure.sequences(MIXED)
    expected = seqs.attend(q, k, v, head_dim=dim)
    after = [c.clone() for c in held]
    over = seqs.attend(q, k, v, head_dim=dim, cache=after, past=past)
    T = q.size(1)
    for shift in (1, 2, 8):
        wide = torch.full((T, M, (H + 2 * G) * dim + 2 * shift), 9.0, dtype=dt, device="cuda")
        parts, at = [], shift
        for t in (q, k, v):
            view = wide[:, :, at:at + t.size(2)].transpose(0, 1)
            view.copy_(t)
            parts.append(view)
            at += t.size(2)
        out = torch.full((T, M, H * dim + 3), 5.0, dtype=dt, device="cuda")
        got = seqs.attend(*parts, head_dim=dim, out=out[:, :, 1:1 + H * dim].transpose(0, 1))
        assert torch.equal(got, expected)
        assert bool((out[:, :, 0] == 5).all()) and bool((out[:, :, 1 + H * dim:] == 5).all())
        # keys beside values in one buffer, sequences inside rows
        both = torch.full((M, 720, len(MIXED), 2 * G * dim + 3 * shift), 4.0, dtype=dt, device="cuda")
        views = [both[..., shift + i * G * dim:shift + (i + 1) * G * dim].transpose(1, 2) for i in range(2)]
        for view, c in zip(views, held):
            view.copy_(c)
        assert torch.equal(seqs.attend(*parts, head_dim=dim, cache=views, past=past), over)
        for view, c in zip(views, after):
            assert torch.equal(view, c)
        assert bool((both[..., :shift] == 4).all()) and bool((both[..., shift + 2 * G * dim:] == 4).all())
        turned = seqs.rotate(parts[0], parts[1], torch.ones(dim // 2, device="cuda"), head_dim=dim, norm="layer")
        plain = seqs.rotate(q, k, torch.ones(dim // 2, device="cuda"), head_dim=dim, norm="layer")
        assert torch.equal(turned[0], plain[0]) and torch.equal(turned[1], plain[1])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_what_mutants_share(mure, dtype):
    """Shared keys, values and caches give every mutant what its own copies would."""
    say(f"[shared] {dtype}")
    dim, H, G, M, dt = 64, 6, 2, 5, TYPES[dtype]
    q, k, v = cuda(*qkv(6, MIXED, H, G, dim, dt, M, own=False))
    past = torch.tensor([5, 2200, 0, 600, 4, 1500, 1030, 0, 511, 1023], dtype=torch.int32).cuda()
    held = cuda(*caches(7, len(MIXED), 2600, G * dim, dt))
    seqs = mure.sequences(MIXED)
    each = [t.expand(M, -1, -1).contiguous() for t in (k, v)]
    assert torch.equal(seqs.attend(q, k[0], v[0], head_dim=dim), seqs.attend(q, *each, head_dim=dim))
    copies = [c.repeat(M, 1, 1, 1) for c in held]
    expected = seqs.attend(q, *each, head_dim=dim, cache=copies, past=past)
    shared = [c[0].clone() for c in held]
    assert torch.equal(seqs.attend(q, k[0], v[0], head_dim=dim, cache=shared, past=past), expected)
    for c, copy in zip(shared, copies):
        assert torch.equal(c.expand(M, -1, -1, -1), copy)
    # shared keys that go to caches of each mutant
    copies = [c.repeat(M, 1, 1, 1) for c in held]
    assert torch.equal(seqs.attend(q, k[0], v[0], head_dim=dim, cache=copies, past=past), expected)
    # shared queries
    one = seqs.attend(q[0], *each, head_dim=dim)
    assert torch.equal(one, seqs.attend(q[:1].expand(M, -1, -1).contiguous(), *each, head_dim=dim))


def test_batches_of_no_tokens(mure):
    say("[empty]")
    z = lambda *s: torch.zeros(*s, device="cuda")  # noqa: E731
    for lengths in ([0], [0, 0, 0]):
        seqs = mure.sequences(lengths)
        cache, past = (z(len(lengths), 4, 8) + 3, z(len(lengths), 4, 8) + 3), z(len(lengths)).int()
        assert seqs.attend(z(2, 0, 16), z(0, 8), z(0, 8), head_dim=8, cache=cache, past=past).shape == (2, 0, 16)
        assert seqs.rotate(z(0, 16), z(0, 8), z(4), head_dim=8)[1].shape == (0, 8)
        assert bool((cache[0] == 3).all()) and bool((cache[1] == 3).all())
    assert mure.gated(z(0, 8), z(4, 8), z(4, 8)).shape == (0, 4)


def test_rows_behind_the_last_sequence(mure):
    """A buffer of more rows than tokens: those behind stay, whatever they hold."""
    say("[behind]")
    lengths, dim = [33, 5, 64, 200], 32
    n = sum(lengths)
    q, k, v = cuda(*qkv(8, [n + 90], 2, 1, dim, torch.bfloat16))
    for t in (q, k, v):
        t[:, n:] = float("nan")
    out = torch.full((n + 90, 2 * dim), 3.0, dtype=torch.bfloat16, device="cuda")
    seqs = mure.sequences(lengths)
    seqs.attend(q[0, :n], k[0, :n], v[0, :n], head_dim=dim, out=out[:n])
    assert bool((out[n:] == 3).all()) and bool(out[:n].isfinite().all())
    seqs.rotate(q[0, :n], None, torch.ones(16, device="cuda"), head_dim=dim, q_out=out[:n])
    assert bool((out[n:] == 3).all()) and bool(out[:n].isfinite().all())
    w = torch.ones(2 * dim, dim, dtype=torch.bfloat16, device="cuda")
    mure.gated(q[0, :n, :dim], w, w + 0, out=out[:n])
    assert bool((out[n:] == 3).all()) and bool(out[:n].isfinite().all())


# ---------------------------------------------------------------- together

@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_prompt_and_tokens_after_it(mure, dtype):
    """A prompt, then tokens one at a time and three at once, each rotated and attended over the cache: the rows of the
    whole sequences, within the bounds of both."""
    say(f"[after] {dtype}")
    dt, dim, H, G, lengths, steps = TYPES[dtype], 48, 4, 2, [20, 3, 600, 129], [1, 1, 3, 1, 18]
    total = [n + sum(steps) for n in lengths]
    q, k, v = cuda(*qkv(9, total, H, G, dim, dt))
    f = (100.0 ** (-torch.arange(24) / 24)).cuda()
    turned_q, turned_k = mure.sequences(total).rotate(q, k, f, head_dim=dim, norm="rms")
    value, bound = R.attend(turned_q.cpu(), turned_k.cpu(), v.cpu(), total, dim)[0]
    cache = [torch.full((4, max(total), G * dim), float("nan"), dtype=dt, device="cuda") for _ in range(2)]
    past = torch.zeros(4, dtype=torch.int32, device="cuda")
    begin = [0] * 4
    for count in [lengths] + [[n] * 4 for n in steps]:
        rows = torch.cat([torch.arange(s + b, s + b + n) for s, b, n in zip(starts(total), begin, count)])
        seqs = mure.sequences(count)
        a, b = seqs.rotate(q[0, rows], k[0, rows], f, head_dim=dim, norm="rms", past=past)
        assert torch.equal(a, turned_q[0, rows]) and torch.equal(b, turned_k[0, rows])
        out = seqs.attend(a, b, v[0, rows], head_dim=dim, cache=cache, past=past)
        R.close(out[None], (value[:, rows], bound[:, rows]), f"{count}")
        past += torch.tensor(count, dtype=torch.int32, device="cuda")
        begin = [x + n for x, n in zip(begin, count)]


def block(mure, seqs, h, w, past=None, cache=None):
    """Norm, projections, rotation, attention, projection, norm, gated layer, projection."""
    _, x = mure.block_norm(h, before="rms", before_weight=w["norm"], residual_out=False)
    q, k, v = ((x @ w[n]) for n in ("q", "k", "v"))
    q, k = seqs.rotate(q, k, w["f"], head_dim=32, norm="rms", q_weight=w["qn"], past=past)
    y = seqs.attend(q, k, v, head_dim=32, cache=cache, past=past)
    h, x = mure.block_norm(y @ w["o"], h, before="rms", before_weight=w["norm"])
    return h + mure.gated(x, w["gate"], w["up"]) @ w["down"]


def weights(seed, width, inner, dt):
    g = torch.Generator().manual_seed(seed)
    w = {n: normal(g, *s, dtype=dt, std=s[0] ** -0.5) for n, s in
         {"q": (width, 128), "k": (width, 64), "v": (width, 64), "o": (128, width), "down": (inner, width)}.items()}
    w.update({n: normal(g, inner, width, dtype=dt, std=width ** -0.5) for n in ("gate", "up")})
    w.update(norm=normal(g, width, mean=1, std=0.1), qn=normal(g, 32, mean=1, std=0.1), f=torch.rand(16, generator=g))
    return {n: t.cuda() for n, t in w.items()}


def test_a_block_against_float64(mure):
    """A run of the operators as a network's block has them: float32, its largest error against the same chain in float64."""
    say("[block]")
    lengths = [12, 1, 90, 33]
    w = weights(10, 96, 160, torch.float32)
    h = normal(torch.Generator().manual_seed(11), sum(lengths), 96)
    got = block(mure, mure.sequences(lengths), h.cuda(), w)
    c = {n: t.double().cpu() for n, t in w.items()}
    norm = lambda x, weight: x * torch.rsqrt((x * x).mean(-1, keepdim=True) + 1e-5) * weight  # noqa: E731
    x = norm(h.double(), c["norm"])
    q = R.rotate((x @ c["q"])[None], c["f"][None], lengths, 32, "rms", c["qn"][None])[0]
    k = R.rotate((x @ c["k"])[None], c["f"][None], lengths, 32, "rms")[0]
    scale = 32 ** -0.5
    y = torch.zeros(136, 128, dtype=torch.float64)
    for s, n in zip(starts(lengths), lengths):
        for head in range(4):
            a, b, z = q[0, s:s + n, head * 32:][:, :32], k[0, s:s + n, head // 2 * 32:][:, :32], (x @ c["v"])[s:s + n, head // 2 * 32:][:, :32]
            p = (a @ b.T * scale).masked_fill(torch.ones(n, n).triu(1).bool(), float("-inf")).softmax(-1)
            y[s:s + n, head * 32:(head + 1) * 32] = p @ z
    e = h.double() + y @ c["o"]
    x = norm(e, c["norm"])
    e = e + (torch.nn.functional.silu(x @ c["gate"].T) * (x @ c["up"].T)) @ c["down"]
    # five products of at most 160 terms one after the other, each relative to sums of their terms' sizes (at most about 10
    # times the results), and a few roundings between: 5 * 160 * 10 units of the largest value at the most
    assert float((got.cpu() - e).abs().max()) <= 8000 * R.U * float(e.abs().max())


# ---------------------------------------------------------------- graphs and streams

def capture(stream, call):
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        out = call()
    return graph, out


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_captured_step_goes_on(own, dtype):
    """One token for each sequence, captured before any other call, over caches that grow: every replay equals the direct call."""
    say(f"[graph step] {dtype}")
    m, side = own
    dt, dim, H, G, n, capacity = TYPES[dtype], 64, 8, 2, 5, 1500
    q, k, v = cuda(*qkv(12, [n], H, G, dim, dt))
    held = cuda(*caches(13, n, capacity, G * dim, dt))
    f = torch.rand(32).cuda()
    w = cuda(normal(torch.Generator().manual_seed(1), 96, H * dim, dtype=dt, std=0.05))[0]
    up = w.flip(0).contiguous()
    start = torch.tensor([0, 510, 1400, 1023, 7], dtype=torch.int32).cuda()
    past, cache = start.clone(), [c.clone() for c in held]
    seqs = m.sequences([1] * n)
    torch.cuda.synchronize()

    def step(past, cache, add):
        a, b = seqs.rotate(q, k, f, head_dim=dim, past=past)
        y = seqs.attend(a, b, v, head_dim=dim, cache=cache, past=past)
        if add:
            past.add_(1)
        return m.gated(y, w, up)

    graph, out = capture(side, lambda: step(past, cache, True))
    direct = [c.clone() for c in held]
    for i in range(6):
        graph.replay()
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            expected = step(start + i, direct, False)
            side.synchronize()
        assert torch.equal(out, expected), i
        assert all(torch.equal(a, b) for a, b in zip(cache, direct)), i
    assert torch.equal(past, start + 6)


def test_graphs_beside_each_other(own):
    say("[graphs beside]")
    m, side = own
    dim, lengths = 64, [1, 1, 300, 17, 4]
    past = torch.tensor([3000, 5, 1100, 2048, 777], dtype=torch.int32).cuda()
    held = cuda(*caches(14, 5, 3400, 2 * dim, torch.bfloat16))
    ps = [cuda(*qkv(15 + i, lengths, 4, 2, dim, torch.bfloat16)) for i in range(3)]
    cs = [[c.clone() for c in held] for _ in range(4)]
    seqs = m.sequences(lengths)
    torch.cuda.synchronize()

    def run(i, j=None):
        return seqs.attend(*ps[i], head_dim=dim, cache=cs[i if j is None else j], past=past)

    with torch.cuda.stream(side):
        expected = [run(i) for i in range(3)]
        side.synchronize()
    first, out1 = capture(side, lambda: (run(0),))
    second, out2 = capture(side, lambda: (run(1), run(2)))      # these two share a workspace, one after the other
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    for i in range(20):
        for t in out1 + out2:
            t.zero_()
        torch.cuda.synchronize()
        with torch.cuda.stream(a):
            first.replay()
        with torch.cuda.stream(b):
            second.replay()
        with torch.cuda.stream(side):
            direct = run(2, 3)
        torch.cuda.synchronize()
        for got, e in zip(out1 + out2 + (direct,), expected + [expected[2]]):
            assert torch.equal(got, e), i


def test_contexts_on_other_streams():
    """Each context works on the stream it was made on, after what that stream holds, beside the other's."""
    say("[streams]")
    lengths, dim = [500, 33, 1], 64
    q, k, v = cuda(*qkv(20, lengths, 4, 2, dim, torch.bfloat16))
    streams = [torch.cuda.Stream() for _ in range(2)]
    made = []
    torch.cuda.synchronize()
    for s in streams:
        with torch.cuda.stream(s):
            made.append(Mure(device=0))
    seqs = [m.sequences(lengths) for m in made]
    for i in range(10):
        outs = []
        for s, b in zip(streams, seqs):
            with torch.cuda.stream(s):
                moved = q + i                       # made on this stream, just before
                outs.append(b.attend(moved, k, v, head_dim=dim))
        torch.cuda.synchronize()
        assert torch.equal(outs[1], outs[0]), i
    torch.cuda.synchronize()
    R.close(outs[0], R.attend((q + 9).cpu(), k.cpu(), v.cpu(), lengths, dim)[0], "out")
    for m in made:
        m.close()


def test_errors_of_other_calls(mure):
    say("[errors]")
    with open("/proc/self/maps") as f:
        hip = C.CDLL(next(line.split()[-1] for line in f if "libamdhip64" in line))
    lengths, dim = [600, 3], 32
    q, k, v = cuda(*qkv(21, lengths, 2, 1, dim, torch.float32))
    held = cuda(*caches(22, 2, 2000, dim, torch.float32))
    past = torch.tensor([1100, 20], dtype=torch.int32).cuda()
    f, w, w2 = torch.rand(16).cuda(), torch.randn(40, 64).cuda(), torch.randn(40, 64).cuda()
    seqs = mure.sequences(lengths)
    y, u = torch.empty_like(q), torch.empty(1, 603, 40, device="cuda")       # torch's own allocations would find the error
    calls = [lambda: seqs.rotate(q, None, f, head_dim=dim, q_out=y)[0], lambda: seqs.attend(q, k, v, head_dim=dim, out=y),
             lambda: seqs.attend(q, k, v, head_dim=dim, cache=held, past=past, out=y), lambda: mure.gated(q, w, w2, out=u)]
    expected = [call().clone() for call in calls]
    torch.cuda.synchronize()
    for call, e in zip(calls, expected):
        p = C.c_void_p()
        assert hip.hipMalloc(C.byref(p), C.c_size_t(1 << 60)) == 2
        try:
            got = call()
        finally:
            hip.hipGetLastError()
        torch.cuda.synchronize()
        assert torch.equal(got, e)


def test_results_raise_the_version(mure):
    say("[versions]")
    rows = lambda *s: torch.ones(*s, device="cuda")  # noqa: E731
    seqs = mure.sequences([4, 3])
    q, k, v, f, w = rows(7, 8), rows(7, 8), rows(7, 8), rows(2), rows(6, 8)
    keys, values = rows(2, 9, 8), rows(2, 9, 8)
    calls = {"rotate q_out": (rows(7, 8), lambda t: seqs.rotate(q, k, f, head_dim=4, q_out=t)),
             "rotate in place": (rows(7, 8), lambda t: seqs.rotate(t, None, f, head_dim=4, q_out=t)),
             "rotate k_out": (rows(7, 8), lambda t: seqs.rotate(q, k, f, head_dim=4, k_out=t)),
             "attend out": (rows(7, 8), lambda t: seqs.attend(q, k, v, head_dim=4, out=t)),
             "cache of keys": (rows(2, 9, 8), lambda t: seqs.attend(q, k, v, head_dim=4, cache=(t, values))),
             "cache of values": (rows(2, 9, 8), lambda t: seqs.attend(q, k, v, head_dim=4, cache=(keys, t))),
             "gated out": (rows(7, 6), lambda t: mure.gated(q, w, w + 0, out=t))}
    for name, (t, call) in calls.items():
        for more in (1, 2):
            call(t)
            assert t._version == more, name
    assert all(t._version == 0 for t in (q, k, v, f, w))
    with pytest.raises(MureError, match="overlaps"):
        seqs.attend(q, k, v, head_dim=4, out=q)
    assert q._version == 0
    # both from one buffer, which each call changes
    both = rows(2, 9, 16)
    seqs.attend(q, k, v, head_dim=4, cache=(both[..., :8], both[..., 8:]))
    assert both._version >= 1


# ---------------------------------------------------------------- large

@pytest.mark.parametrize("count,past", [(1, 39000), (16, 38500), (40, 39900), (600, 39000)])
def test_a_cache_of_more_bytes_than_32_bits(mure, count, past):
    """5.2 GB for a sequence's keys and values each, of which the last rows lie behind 2^32 bytes."""
    say(f"[large cache] {count} {past}")
    dim, rows, wide = 64, 40000, 1 << 16
    g = torch.Generator(device="cuda").manual_seed(30)
    cache = []
    for _ in range(2):
        whole = torch.empty(1, rows, wide, dtype=torch.bfloat16, device="cuda")
        view = whole[:, :, wide - dim:]
        view.copy_(torch.randn(1, rows, dim, generator=g, device="cuda"))
        cache.append(view)
    q, k, v = qkv(31, [count], 2, 1, dim, torch.bfloat16)
    p = torch.tensor([past], dtype=torch.int32)
    held = [c[None].cpu() for c in cache]
    window = None if count <= 16 else 300               # the reference has a product for every token and key
    out = mure.sequences([count]).attend(*cuda(q, k, v), head_dim=dim, cache=cache, past=p.cuda(), window=window)
    if window:                                          # only the keys that anyone sees
        first = past - window
        value = R.attend(q, k, v, [count], dim, window=window, cache=[c[:, :, first:] for c in held], past=torch.tensor([window]))[0]
    else:
        value = R.attend(q, k, v, [count], dim, cache=held, past=p)[0]
    R.close(out, value, "out")
    for c, h, new in zip(cache, held, (k, v)):
        h[:, :, past:past + count] = new
        assert torch.equal(c.cpu(), h[0])


def test_tensors_of_more_bytes_than_32_bits(mure):
    """Rows behind 2^32 bytes of q, out and a gated layer's tensors: those of the last sequence alone."""
    say("[large tensors]")
    dim, H, lengths = 64, 128, [100] * 2799 + [67, 300, 5]
    T = sum(lengths)
    g = torch.Generator(device="cuda").manual_seed(32)
    q = torch.randn(T, H * dim, generator=g, device="cuda", dtype=torch.bfloat16)
    k, v = (torch.randn(T, 2 * dim, generator=g, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    assert q.numel() * 2 > 1 << 32
    f = torch.rand(32, generator=g, device="cuda")
    seqs, last, one = mure.sequences(lengths), slice(T - 372, T), mure.sequences(lengths[-3:])
    expected = one.rotate(q[last], None, f, head_dim=dim, norm="rms")[0]
    out = torch.empty_like(q)
    seqs.rotate(q, None, f, head_dim=dim, norm="rms", q_out=out)
    assert torch.equal(out[last], expected)
    seqs.attend(q, k, v, head_dim=dim, out=out)
    assert torch.equal(out[last], one.attend(q[last], k[last], v[last], head_dim=dim))
    assert torch.equal(out[:100], mure.sequences([100]).attend(q[:100], k[:100], v[:100], head_dim=dim))
    w = torch.randn(H * dim, 32, generator=g, device="cuda", dtype=torch.bfloat16)
    mure.gated(q[:, -32:], w, w.flip(0), out=out)
    assert torch.equal(out[last], mure.gated(q[last, -32:], w, w.flip(0)))


def test_many_sequences_and_mutants(mure):
    """More blocks than a launch has, in every kernel: 12 million sequences of one and two tokens, of one head of two channels."""
    say("[many]")
    M, n, dim = 600, 20000, 2
    lengths = [1, 2] * (n // 2)
    T = sum(lengths)
    g = torch.Generator(device="cuda").manual_seed(33)
    q, k, v = (torch.randn(M, T, dim, generator=g, device="cuda") for _ in range(3))
    seqs = mure.sequences(lengths)
    f = torch.ones(1, device="cuda")
    a, _ = seqs.rotate(q, None, f, head_dim=dim)
    out = seqs.attend(q, k, v, head_dim=dim)
    one = mure.sequences([1, 2])
    for m in (0, 299, M - 1):
        at = (m, slice(T - 3, T))
        assert torch.equal(a[at], one.rotate(q[at], None, f, head_dim=dim)[0])
        assert torch.equal(out[at], one.attend(q[at], k[at], v[at], head_dim=dim))
    # a single token's result is its value, (v w) (1 / w) with any w: three roundings of a unit each
    for at in (0, 3):
        assert bool(((out[:, at] - v[:, at]).abs() <= 3.01 * R.U * v[:, at].abs()).all())
    cache = [torch.randn(M, n, 3, dim, generator=g, device="cuda") for _ in range(2)]
    past = torch.ones(n, dtype=torch.int32, device="cuda")
    before = [c[M - 1, n - 2:].clone() for c in cache]
    out = seqs.attend(q, k, v, head_dim=dim, cache=cache, past=past)
    at = (M - 1, slice(T - 3, T))
    assert torch.equal(out[at], one.attend(q[at], k[at], v[at], head_dim=dim, cache=before, past=past[:2]))
    assert all(torch.equal(c[M - 1, n - 2:], b) for c, b in zip(cache, before))


def test_parts_of_many_sequences_over_a_long_cache(mure):
    """Parts that take more workspace than a call has: some sequences after the others, each as it is alone."""
    say("[parts]")
    dim, H, capacity, lengths = 64, 32, 131072, [300, 16, 512, 17, 3, 260, 1, 512]
    g = torch.Generator(device="cuda").manual_seed(40)
    T, n = sum(lengths), len(lengths)
    q = torch.randn(2, T, H * dim, generator=g, device="cuda", dtype=torch.bfloat16)
    k, v = (torch.randn(2, T, dim, generator=g, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    cache = [torch.randn(2, n, capacity, dim, generator=g, device="cuda", dtype=torch.bfloat16) for _ in range(2)]
    past = torch.tensor([3000, 130000, 1024, 5000, 70000, 1, 2000, 4090], dtype=torch.int32, device="cuda")
    before = [c.clone() for c in cache]
    out = mure.sequences(lengths).attend(q, k, v, head_dim=dim, cache=cache, past=past)
    assert bool(out.isfinite().all())
    for i, (s, count) in enumerate(zip(starts(lengths), lengths)):
        for m in (0, 1):
            at = (m, slice(s, s + count))
            alone = mure.sequences([count]).attend(q[at], k[at], v[at], head_dim=dim, cache=[b[m, i:i + 1] for b in before], past=past[i:i + 1])
            assert torch.equal(out[at], alone), (i, m)
    assert all(torch.equal(c, b) for c, b in zip(cache, before))
    # a window wider than 64 bits' half
    wide = mure.sequences([40]).attend(q[0, :40], k[0, :40], v[0, :40], head_dim=dim, causal=False, window=(1 << 63) - 1)
    assert torch.equal(wide, mure.sequences([40]).attend(q[0, :40], k[0, :40], v[0, :40], head_dim=dim, causal=False))
