"""The operators of a selective state space block on the GPU, against their
definitions in float64 with running rounding bounds (``seq_reference``)."""
import random

import pytest
import torch

import seq_reference as R
from paper_2607_18582_amd import Mure, MureError

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
RAGGED = [5, 0, 1, 33, 2, 64, 3, 31, 0]


@pytest.fixture(scope="module")
def mure():
    m = Mure(device=0)
    yield m
    m.close()


def say(*a):
    print(*a, flush=True)


def normal(g, *shape, dtype=torch.float32, mean=0.0, std=1.0):
    """On the CPU, already rounded to dtype."""
    return (torch.randn(*shape, generator=g) * std + mean).to(dtype)


def cuda(*tensors):
    return [None if t is None else t.cuda() for t in tensors]


# ---------------------------------------------------------------- convolution

def conv_inputs(seed, lengths, C, K, dtype, M=1, own=False, bias=True, state=False):
    g = torch.Generator().manual_seed(seed)
    T, n = sum(lengths), len(lengths)
    x = normal(g, M if own else 1, T, C, dtype=dtype)
    taps = normal(g, M, C, K, dtype=dtype, std=K ** -0.5)
    b = normal(g, M, C, std=0.2) if bias else None
    st = normal(g, M if own else 1, n, K - 1, C, dtype=dtype) if state else None
    return x, taps, b, st


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("C,K,M,own,bias,state,act", [
    (1, 4, 1, False, True, True, "silu"), (3, 2, 2, True, False, False, None), (8, 1, 1, False, True, False, "silu"),
    (17, 3, 3, False, True, True, None), (64, 4, 1, False, True, False, "silu"), (129, 5, 2, True, True, True, "silu"),
    (100, 6, 1, False, False, True, None), (260, 7, 2, False, True, True, "silu"), (7, 8, 1, False, True, True, "silu"),
    (512, 4, 5, False, True, False, "silu")])
def test_conv(mure, dtype, C, K, M, own, bias, state, act):
    say(f"[conv] {dtype} C={C} K={K} M={M}")
    x, taps, b, st = conv_inputs(C + K, RAGGED, C, K, TYPES[dtype], M, own, bias, state)
    seqs = mure.sequences(RAGGED)
    gx, gt, gb, gs = cuda(x, taps, b, st)
    y, last = seqs.conv(gx, gt, gb, activation=act, state=gs)
    ey, el = R.conv(x, taps, b, RAGGED, act, st)
    R.close(y, ey, "out")
    assert torch.equal(last.cpu().double(), el[0])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_conv_resumed_is_the_whole(mure, dtype):
    """Prompts in two parts and then token by token, the state updated in place, give the whole's bits."""
    say(f"[conv resumed] {dtype}")
    lengths, C, K = [40, 9, 3], 72, 4
    x, taps, b, _ = cuda(*conv_inputs(1, lengths, C, K, TYPES[dtype]))
    whole, last = mure.sequences(lengths).conv(x[0], taps[0], b[0], activation="silu")
    start = [0, 40, 49]
    done, state = [0, 0, 0], torch.zeros(3, K - 1, C, dtype=x.dtype, device="cuda")
    for part in ([17, 2, 0], [20, 0, 2]) + ([1, 1, 0],) * 2 + ([0, 1, 1],) + ([1, 1, 0],) + ([0, 1, 0],) * 3:
        rows = torch.cat([x[0, s + d:s + d + p] for s, d, p in zip(start, done, part)])
        y, same = mure.sequences(part).conv(rows, taps[0], b[0], activation="silu", state=state, state_out=state)
        assert same is state
        at = 0
        for s, d, p in zip(start, done, part):
            assert torch.equal(y[at:at + p], whole[s + d:s + d + p])
            at += p
        done = [d + p for d, p in zip(done, part)]
    assert done == lengths
    assert torch.equal(state, last)


@pytest.mark.parametrize("K", range(2, 9))
def test_conv_updates_states_in_place(mure, K):
    """Short sequences of every number of taps: every run has read the old state before it is overwritten."""
    say(f"[conv in place] K={K}")
    lengths, C = [11, 1, 8, 0, 3, 40, 4, 5], 24
    x, taps, b, st = conv_inputs(K, lengths, C, K, torch.bfloat16, state=True)
    seqs = mure.sequences(lengths)
    y, last = seqs.conv(*cuda(x, taps, b), state=st.cuda())
    R.close(y, R.conv(x, taps, b, lengths, None, st)[0], "out")
    for _ in range(20):
        held = st.cuda()
        y2, same = seqs.conv(*cuda(x, taps, b), state=held, state_out=held)
        assert same is held and torch.equal(y2, y) and torch.equal(held, last)


def test_conv_strided_views(mure):
    """Rows that are slices of wider ones, at odd addresses, in and out, and an expanded mutant axis."""
    say("[conv strided]")
    lengths, C, K, M = [7, 20], 37, 4, 3
    x, taps, b, _ = conv_inputs(2, lengths, C, K, torch.bfloat16, M, own=False)
    wide = torch.full((27, 2 * C + 3), 9.0, dtype=torch.bfloat16, device="cuda")
    wide[:, 3:3 + C] = x[0].cuda()
    into = torch.full((M, 27, C + 5), 7.0, dtype=torch.bfloat16, device="cuda")
    y, _ = mure.sequences(lengths).conv(wide[:, 3:3 + C].expand(M, 27, C), taps.cuda(), b.cuda(), out=into[..., 1:1 + C])
    assert y.data_ptr() == into[..., 1:].data_ptr()
    R.close(y, R.conv(x, taps, b, lengths)[0], "out")
    assert bool((into[..., 0] == 7).all()) and bool((into[..., 1 + C:] == 7).all())
    # out beside x in the same rows
    both = torch.zeros(27, 2 * C, dtype=torch.bfloat16, device="cuda")
    both[:, :C] = x[0].cuda()
    y2, _ = mure.sequences(lengths).conv(both[:, :C], taps[0].cuda(), b[0].cuda(), out=both[:, C:])
    assert torch.equal(y2, y[0]) and torch.equal(both[:, :C], x[0].cuda())


def test_conv_infinities_stay_in_their_sequence_and_window(mure):
    say("[conv inf]")
    lengths, C, K = [9, 9], 16, 3
    x, taps, b, _ = conv_inputs(3, lengths, C, K, torch.float32)
    x[0, 4, 2], x[0, 5, 3], x[0, 8, 5] = float("inf"), float("nan"), float("-inf")
    taps[0, 6] = 0
    x[0, 12, 6] = float("inf")                  # 0 times infinity: NaN, as by the definition
    y, last = mure.sequences(lengths).conv(*cuda(x, taps, b), activation="silu")
    ey, el = R.conv(x, taps, b, lengths, "silu")
    R.close(y, ey, "out")                       # silu(-inf) = -inf / inf: NaN by the formula too
    assert torch.equal(last.cpu().double().nan_to_num(5), el[0].nan_to_num(5))


# ---------------------------------------------------------------- scan

def scan_inputs(seed, lengths, D, N, dtype, G=1, M=1, own=True, gate=True, state=False, mutated=False):
    g = torch.Generator().manual_seed(seed)
    T, n, mo, mp = sum(lengths), len(lengths), M if own else 1, M if mutated else 1
    step = torch.exp(torch.rand(mp, D, generator=g) * 4.6 - 6.9)
    return dict(u=normal(g, mo, T, D, dtype=dtype), dt=normal(g, mo, T, D, dtype=dtype, std=0.5),
                A=-torch.arange(1, N + 1) * torch.exp(normal(g, mp, D, N, std=0.3)),
                B=normal(g, mo, T, G * N, dtype=dtype), C=normal(g, mo, T, G * N, dtype=dtype),
                skip=normal(g, mp, D, mean=1.0), dt_bias=step + torch.log(-torch.expm1(-step)),
                gate=normal(g, mo, T, D, dtype=dtype) if gate else None,
                state=normal(g, mo, n, D, N) if state else None)


def run_scan(seqs, p, **more):
    q = {k: None if v is None else v.cuda() for k, v in p.items()}
    return seqs.scan(q["u"], q["dt"], q["A"], q["B"], q["C"], skip=q["skip"], dt_bias=q["dt_bias"], gate=q["gate"],
                     state=q["state"], **more)


def check_scan(mure, p, lengths, **more):
    y, last = run_scan(mure.sequences(lengths), p, **more)
    ey, el = R.scan(p["u"], p["dt"], p["A"], p["B"], p["C"], lengths, p["skip"], p["dt_bias"], p["gate"],
                    more.get("softplus", True), p["state"])
    say("   worst:", R.close(y, ey, "out"), R.close(last, el, "state"))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("D,N,G,M,own,mutated,gate,state", [
    (1, 1, 1, 1, True, False, True, True), (16, 16, 1, 1, True, False, True, False), (5, 2, 1, 2, True, False, False, True),
    (64, 4, 2, 1, True, False, True, True), (70, 5, 1, 2, False, True, True, False), (33, 8, 3, 1, True, False, True, True),
    (130, 16, 1, 3, False, True, True, True), (48, 17, 4, 1, True, False, True, False), (20, 32, 1, 1, True, False, False, True),
    (66, 33, 2, 1, True, False, True, True), (40, 64, 1, 2, True, True, True, True)])
def test_scan(mure, dtype, D, N, G, M, own, mutated, gate, state):
    say(f"[scan] {dtype} D={D} N={N} G={G} M={M}")
    check_scan(mure, scan_inputs(D + N, RAGGED, D, N, TYPES[dtype], G, M, own, gate, state, mutated), RAGGED)


@pytest.mark.parametrize("dtype,lengths,D,N,state", [
    ("f32", [1024, 1025, 0, 1], 20, 16, True), ("bf16", [1300, 7, 2049], 12, 6, False), ("f32", [4097], 8, 16, True),
    ("bf16", [1024 + 128 * 3], 70, 4, True)])
def test_scan_in_chunks(mure, dtype, lengths, D, N, state):
    say(f"[scan chunks] {dtype} {lengths}")
    check_scan(mure, scan_inputs(7, lengths, D, N, TYPES[dtype], state=state, M=2, own=True), lengths)


def test_scan_without_softplus_and_options(mure):
    say("[scan options]")
    p = scan_inputs(8, RAGGED, 24, 16, torch.float32)
    p["dt"] = p["dt"].abs() * 0.1
    p["dt_bias"] = p["skip"] = None
    check_scan(mure, p, RAGGED, softplus=False)
    p["dt"] = p["dt"] * 0                       # a step of 0 keeps the state and adds nothing
    p["state"] = normal(torch.Generator().manual_seed(1), 1, len(RAGGED), 24, 16)
    y, last = run_scan(mure.sequences(RAGGED), p, softplus=False)
    assert torch.equal(last.cpu(), p["state"])


def test_scan_extreme_values(mure):
    """Steps from vanishing to huge, rates of 0, positive, and -inf; each in channels of its own."""
    say("[scan extremes]")
    lengths, N = [6, 3], 5
    p = scan_inputs(9, lengths, 64, N, torch.float32, state=True)
    p["dt"][0, :, 0] = -80.0                    # softplus below the smallest float32 but for its tail
    p["dt"][0, :, 1] = 60.0
    p["dt"][0, :, 2] = float("-inf")            # a step of exactly 0
    p["A"][0, 3] = 0.0
    p["A"][0, 4] = 0.5
    p["A"][0, 5] = float("-inf")                # forgets at once
    p["A"][0, 6, 4] = float("-inf")
    p["dt"][0, :, 7] = -16.0                    # e^s below a float32's unit: log1p must keep it
    p["state"][0, 1, 8] = 1e30
    check_scan(mure, p, lengths)


@pytest.mark.parametrize("N", [3, 16])
def test_scan_infinities_stay_in_their_channel_and_sequence(mure, N):
    say(f"[scan inf] N={N}")
    lengths, D = [5, 0, 6], 40
    p = scan_inputs(10, lengths, D, N, torch.float32)
    p["B"] = p["B"].abs() + 0.1                 # so that infinite inputs give infinite states, all of one sign
    p["C"] = p["C"].abs() + 0.1
    p["gate"] = None
    p["u"][0, 2, 3] = float("inf")
    p["u"][0, 6, 4] = float("nan")
    p["dt"][0, 7, 5] = float("nan")
    p["skip"] = p["skip"].abs()
    check_scan(mure, p, lengths)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_scan_resumed_is_the_whole(mure, dtype):
    say(f"[scan resumed] {dtype}")
    lengths, D, N = [50, 13], 70, 16
    p = scan_inputs(11, lengths, D, N, TYPES[dtype])
    q = {k: None if v is None else v.cuda()[0] for k, v in p.items()}
    whole, last = mure.sequences(lengths).scan(q["u"], q["dt"], q["A"], q["B"], q["C"], skip=q["skip"], dt_bias=q["dt_bias"],
                                               gate=q["gate"])
    start, done, state = [0, 50], [0, 0], torch.zeros(2, D, N, device="cuda")
    for part in ([33, 0], [15, 10], [1, 1], [1, 1], [0, 1]):
        def cut(v):
            return torch.cat([v[s + d:s + d + c] for s, d, c in zip(start, done, part)])
        y, _ = mure.sequences(part).scan(cut(q["u"]), cut(q["dt"]), q["A"], cut(q["B"]), cut(q["C"]), skip=q["skip"],
                                         dt_bias=q["dt_bias"], gate=cut(q["gate"]), state=state, state_out=state)
        at = 0
        for s, d, c in zip(start, done, part):
            assert torch.equal(y[at:at + c], whole[s + d:s + d + c])
            at += c
        done = [d + c for d, c in zip(done, part)]
    assert done == lengths and torch.equal(state, last)


def test_scan_chunks_update_the_state_in_place(mure):
    say("[scan chunks in place]")
    lengths = [1500, 20]
    p = scan_inputs(12, lengths, 24, 16, torch.float32, state=True)
    y, last = run_scan(mure.sequences(lengths), p)
    held = p["state"].cuda()
    q = {k: None if v is None else v.cuda() for k, v in p.items()}
    y2, same = mure.sequences(lengths).scan(q["u"], q["dt"], q["A"], q["B"], q["C"], skip=q["skip"], dt_bias=q["dt_bias"],
                                            gate=q["gate"], state=held, state_out=held)
    assert same is held and torch.equal(held, last) and torch.equal(y2, y)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_results_do_not_depend_on_the_batch(mure, dtype):
    """A sequence alone, a mutant alone, and all together: the same bits."""
    say(f"[batch] {dtype}")
    lengths, D, N, M = [300, 1, 1200, 40], 96, 16, 5
    p = scan_inputs(13, lengths, D, N, TYPES[dtype], M=M, own=True, mutated=True, state=True)
    q = {k: None if v is None else v.cuda() for k, v in p.items()}
    y, last = run_scan(mure.sequences(lengths), p)
    x, taps, b, st = cuda(*conv_inputs(14, lengths, D, 4, TYPES[dtype], M, own=True, state=True))
    yc, lc = mure.sequences(lengths).conv(x, taps, b, activation="silu", state=st)
    row = 0
    for i, n in enumerate(lengths):
        one, m = mure.sequences([n]), (2 * i + 1) % M
        cut = slice(row, row + n)
        ys, ls = one.scan(q["u"][m, cut], q["dt"][m, cut], q["A"][m], q["B"][m, cut], q["C"][m, cut], skip=q["skip"][m],
                          dt_bias=q["dt_bias"][m], gate=q["gate"][m, cut], state=q["state"][m, i:i + 1])
        assert torch.equal(ys, y[m, cut]) and torch.equal(ls[0], last[m, i])
        ys, ls = one.conv(x[m, cut], taps[m], b[m], activation="silu", state=st[m, i:i + 1])
        assert torch.equal(ys, yc[m, cut]) and torch.equal(ls[0], lc[m, i])
        row += n


# ---------------------------------------------------------------- norms

@pytest.mark.parametrize("dtype,residual", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32")])
@pytest.mark.parametrize("width", [1, 7, 8, 100, 128, 257, 512, 1003, 1024, 2048, 2049, 4096, 8200, 16384])
def test_block_norm(mure, dtype, residual, width):
    say(f"[norm] {dtype}/{residual} {width}")
    g = torch.Generator().manual_seed(width)
    rows, M = 5, 2
    y, z = normal(g, M, rows, width, dtype=TYPES[dtype], mean=0.3), normal(g, M, rows, width, dtype=TYPES[dtype])
    r = normal(g, 1, rows, width, dtype=TYPES[residual], std=2.0)
    aw, ab, s, bw, bb = (normal(g, 1 + (i == 2), width, mean=1.0, std=0.2) for i in range(5))
    for options in (dict(after="rms", before="layer", gate=z), dict(after="layer", before="rms", gate=z, gate_at="after", gate_activation="sigmoid"),
                    dict(before="rms"), dict(after="layer"), dict(gate=z, gate_activation=None, before="layer")):
        p = dict(options, residual=r)
        if "after" in p:
            p.update(after_weight=aw, after_bias=ab, scale=s)
        if "before" in p:
            p.update(before_weight=bw, before_bias=bb if "after" in p else None)
        q = {k: v.cuda() if isinstance(v, torch.Tensor) else v for k, v in p.items()}
        ro, out = mure.block_norm(y.cuda(), **q)
        er, eo = R.block_norm(y, **p)
        R.close(ro, er, "residual_out")
        assert ro.dtype == TYPES[residual]
        if eo is None:
            assert out is None
        else:
            R.close(out, eo, "out")


def test_block_norm_forms(mure):
    """Alone before a block, alone after it, in place, one mutant at a time, zero rows, an empty batch of rows."""
    say("[norm forms]")
    g = torch.Generator().manual_seed(3)
    y, r = normal(g, 9, 200, dtype=torch.bfloat16), normal(g, 9, 200)
    gy, gr = y.cuda(), r.cuda()
    none, o = mure.block_norm(gy, before="rms", residual_out=False)
    assert none is None
    R.close(o, tuple(t[0] for t in R.block_norm(y[None], before="rms")[1]), "before")
    ro, o = mure.block_norm(gy, gr, scale=0.25)
    assert o is None and ro.dtype == torch.float32
    R.close(ro, tuple(t[0] for t in R.block_norm(y[None], r[None], scale=0.25)[0]), "sum")
    a, b = mure.block_norm(gy, gr, after="rms", before="layer")
    held, into = gr.clone(), gy.clone()
    ro, o = mure.block_norm(into, held, after="rms", before="layer", residual_out=held, out=into)
    assert ro is held and o is into and torch.equal(held, a) and torch.equal(into, b)
    many = torch.stack([gy, gy * 2, gy * 0])
    am, bm = mure.block_norm(many, gr, after="rms", before="layer")
    assert torch.equal(am[0], a) and torch.equal(bm[0], b)
    assert torch.equal(am[2], gr)               # a row of zeros has a norm of zeros
    empty = mure.block_norm(gy[:0], gr[:0], before="rms")
    assert empty[0].shape == (0, 200) and empty[1].shape == (0, 200)


# ---------------------------------------------------------------- streams, graphs, sizes

def test_other_streams(mure):
    """A call under another current stream waits for it, and it for the call."""
    say("[streams]")
    lengths = [700, 300]
    x, taps, b, _ = cuda(*conv_inputs(15, lengths, 256, 4, torch.float32))
    seqs = mure.sequences(lengths)
    expected, _ = seqs.conv(x[0], taps[0], b[0])
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        late = torch.zeros_like(x[0])
        big = torch.randn(4096, 4096, device="cuda")
        for _ in range(8):
            big = big @ big * 1e-3              # some time before the input is there
        late.copy_(x[0])
        y, _ = seqs.conv(late, taps[0], b[0])
        late.zero_()                            # after the call, on the side stream
        total = y.clone()
    side.synchronize()
    assert torch.equal(total, expected)


def test_graph_replays(mure):
    """A captured block, replayed with new inputs and eager work between the replays."""
    say("[graph]")
    lengths, D, N = [1100, 6, 0, 80], 64, 16
    p = scan_inputs(16, lengths, D, N, torch.float32)
    q = {k: None if v is None else v.cuda()[0] for k, v in p.items()}
    x, taps, b, _ = cuda(*conv_inputs(17, lengths, D, 4, torch.float32))
    x = x[0]
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        own = Mure(device=0)
    seqs = own.sequences(lengths)

    def block():
        u, _ = seqs.conv(x, taps[0], b[0], activation="silu")
        y, _ = seqs.scan(u, q["dt"], q["A"], q["B"], q["C"], skip=q["skip"], dt_bias=q["dt_bias"], gate=q["gate"])
        return own.block_norm(y, x, after="rms", before="layer")

    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        block()                                 # the workspace of its size
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            out = block()
        for i in range(4):
            x.copy_(normal(torch.Generator().manual_seed(i), *x.shape))
            graph.replay()
            got = [t.clone() for t in out]
            eager = block()
            side.synchronize()
            assert all(torch.equal(a, e) for a, e in zip(got, eager)), i
    own.close()


def test_offsets_past_32_bits(mure):
    """Rows and mutants whose elements lie beyond 2^32 bytes and 2^31 elements."""
    say("[offsets]")
    T, C, far = 40, 64, (1 << 31) // 32 + 17
    whole = torch.zeros(40 * far + C, dtype=torch.bfloat16, device="cuda")
    rows = whole.as_strided((T, C), (far, 1))   # the last row starts past 2^31 elements
    x, taps, b, _ = conv_inputs(18, [T], C, 4, torch.bfloat16)
    rows.copy_(x[0].cuda())
    y, _ = mure.sequences([T]).conv(rows, taps[0].cuda(), b[0].cuda(), activation="silu")
    R.close(y[None], R.conv(x, taps, b, [T], "silu")[0], "conv")
    p = scan_inputs(19, [T], C, 16, torch.bfloat16)
    q = {k: None if v is None else v.cuda()[0] for k, v in p.items()}
    rows.copy_(q["u"])
    y, _ = mure.sequences([T]).scan(rows, q["dt"], q["A"], q["B"], q["C"], skip=q["skip"], dt_bias=q["dt_bias"], gate=q["gate"])
    R.close(y[None], R.scan(p["u"], p["dt"], p["A"], p["B"], p["C"], [T], p["skip"], p["dt_bias"], p["gate"])[0], "scan")
    rows.copy_(x[0].cuda())
    r, o = mure.block_norm(rows, before="rms")
    R.close(o[None], R.block_norm(x, before="rms")[1], "norm")
    out, _ = mure.sequences([T]).conv(x[0].cuda(), taps[0].cuda(), b[0].cuda(), activation="silu", out=rows)
    R.close(out[None], R.conv(x, taps, b, [T], "silu")[0], "out")


def test_refusals_on_the_gpu(mure):
    say("[refusals]")
    seqs = mure.sequences([4, 4])
    x = torch.zeros(8, 16, device="cuda")
    taps = torch.zeros(16, 4, device="cuda")
    with pytest.raises(MureError, match="out overlaps x"):
        seqs.conv(x, taps, out=x)
    with pytest.raises(TypeError):
        seqs.conv(x, taps.bfloat16())
    with pytest.raises(TypeError):
        seqs.conv(x, taps.cpu())
    with pytest.raises(ValueError):
        seqs.conv(x[:7], taps)
    with pytest.raises(ValueError):
        seqs.conv(x.cpu(), taps)
    y, _ = seqs.conv(x, taps)                   # and the context goes on working
    assert bool((y == 0).all())
    seqs.close()
    with pytest.raises(ValueError, match="closed"):
        seqs.conv(x, taps)


@pytest.mark.parametrize("seed", range(6))
def test_drawn_sizes(mure, seed):
    """Sizes at random: odd widths, states and lengths together."""
    rng = random.Random(seed)
    lengths = [rng.choice([0, 1, rng.randint(1, 70)]) for _ in range(rng.randint(1, 6))] + [rng.randint(1, 9)]
    dtype, D, N, M = rng.choice(["f32", "bf16"]), rng.randint(1, 150), rng.randint(1, 40), rng.randint(1, 3)
    say(f"[drawn] {dtype} {lengths} D={D} N={N} M={M}")
    check_scan(mure, scan_inputs(seed, lengths, D, N, TYPES[dtype], 1, M, rng.random() < 0.5, rng.random() < 0.5, rng.random() < 0.5,
                                 rng.random() < 0.5), lengths)
    K = rng.randint(1, 8)
    x, taps, b, st = conv_inputs(seed, lengths, D, K, TYPES[dtype], M, rng.random() < 0.5, rng.random() < 0.5, rng.random() < 0.5)
    y, last = mure.sequences(lengths).conv(*cuda(x, taps, b), activation="silu", state=None if st is None else st.cuda())
    ey, el = R.conv(x, taps, b, lengths, "silu", st)
    R.close(y, ey, "conv")
    assert torch.equal(last.cpu().double(), el[0])


@pytest.mark.parametrize("dtype,lengths,D,N,G,state", [
    ("f32", [513, 1030, 3], 2048, 16, 1, True), ("bf16", [700, 512, 0, 1500], 1024, 16, 1, False),
    ("bf16", [1024, 2048], 2052, 5, 4, True), ("f32", [530], 1100, 3, 1, True), ("f32", [600], 2050, 20, 1, True)])
def test_scan_of_wide_layers(mure, dtype, lengths, D, N, G, state):
    """Long sequences of wide layers; a few channels are compared."""
    say(f"[scan wide] {dtype} {lengths} D={D} N={N}")
    p = scan_inputs(20, lengths, D, N, TYPES[dtype], G, state=state)
    p["A"][0, 1] = float("-inf")
    y, last = run_scan(mure.sequences(lengths), p)
    # per group: the first channels, some in the middle and the last
    width = D // G
    some = torch.tensor(sorted({g * width + c for g in range(G) for c in (0, 1, 2, 63, 64, width // 2, width - 2, width - 1)}))
    cut = lambda v, axis: None if v is None else v.index_select(axis, some)  # noqa: E731
    gid = some // width
    spread = lambda v: v.view(1, -1, G, N)[:, :, gid].reshape(1, -1, len(some) * N)  # noqa: E731
    ey, el = R.scan(cut(p["u"], 2), cut(p["dt"], 2), cut(p["A"], 1), spread(p["B"]), spread(p["C"]), lengths, cut(p["skip"], 1),
                    cut(p["dt_bias"], 1), cut(p["gate"], 2), True, cut(p["state"], 2))
    say("   worst:", R.close(y[:, :, some.cuda()], ey, "out"), R.close(last[:, :, some.cuda()], el, "state"))


def test_wide_layers_do_not_depend_on_the_batch(mure):
    say("[scan wide batch]")
    lengths, D, N, M = [520, 20, 1300], 2048, 16, 2
    p = scan_inputs(21, lengths, D, N, torch.bfloat16, M=M, own=True, mutated=True, state=True)
    q = {k: None if v is None else v.cuda() for k, v in p.items()}
    y, last = run_scan(mure.sequences(lengths), p)
    row = 0
    for i, n in enumerate(lengths):
        cut, m = slice(row, row + n), (i + 1) % M
        held = q["state"][m, i:i + 1].clone()
        ys, ls = mure.sequences([n]).scan(q["u"][m, cut], q["dt"][m, cut], q["A"][m], q["B"][m, cut], q["C"][m, cut], skip=q["skip"][m],
                                          dt_bias=q["dt_bias"][m], gate=q["gate"][m, cut], state=held, state_out=held)
        assert torch.equal(ys, y[m, cut]) and torch.equal(ls[0], last[m, i])
        row += n


@pytest.mark.parametrize("D", [16, 1024, 2048])
def test_infinite_states_of_long_sequences(mure, D):
    """An infinite state stays infinite over spans in which any finite one decays to nothing, as token by token."""
    say(f"[scan inf long] D={D}")
    lengths, N = [1300], 16
    p = scan_inputs(22, lengths, D, N, torch.float32)
    p["B"], p["C"], p["skip"], p["gate"] = p["B"].abs() + 0.1, p["C"].abs() + 0.1, p["skip"].abs(), None
    p["dt"][0, :, 3] += 8                       # steps of some 5: a decay of e^-80 a token for the last state
    p["u"][0, 100, 3] = float("inf")
    p["u"][0, 700, 5] = float("nan")
    y, last = run_scan(mure.sequences(lengths), p)
    assert bool(torch.isposinf(y[0, 100:, 3]).all()) and bool(torch.isposinf(last[0, 0, 3]).all())
    assert bool(torch.isnan(y[0, 700:, 5]).all()) and bool(torch.isfinite(y[0, :700, 5]).all())
    rest = [c for c in range(D) if c not in (3, 5)]
    assert bool(torch.isfinite(y[0][:, rest]).all()) and bool(torch.isfinite(last[0, 0][rest]).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_scan_of_rows_far_apart(mure, dtype):
    """Rows of which four span more than 2^32 bytes, read and written."""
    say(f"[scan far rows] {dtype}")
    T, D, N = 7, 70, 16
    far = (1 << 32) // (3 * TYPES[dtype].itemsize) + 101
    whole = torch.empty((T - 1) * far + D, dtype=TYPES[dtype], device="cuda")
    rows = whole.as_strided((T, D), (far, 1))
    p = scan_inputs(23, [T], D, N, TYPES[dtype])
    q = {k: None if v is None else v.cuda()[0] for k, v in p.items()}
    rest = dict(skip=q["skip"], dt_bias=q["dt_bias"], gate=q["gate"])
    seqs = mure.sequences([T])
    expected, last = seqs.scan(q["u"], q["dt"], q["A"], q["B"], q["C"], **rest)
    R.close(expected[None], R.scan(p["u"], p["dt"], p["A"], p["B"], p["C"], [T], p["skip"], p["dt_bias"], p["gate"])[0], "near")
    rows.copy_(q["u"])
    y, state = seqs.scan(rows, q["dt"], q["A"], q["B"], q["C"], **rest)
    assert torch.equal(y, expected) and torch.equal(state, last)
    y, state = seqs.scan(q["u"], q["dt"], q["A"], q["B"], q["C"], out=rows, **rest)
    assert y is rows and torch.equal(rows, expected) and torch.equal(state, last)
