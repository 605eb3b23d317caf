"""Scans of one batch captured into several graphs: the graphs' workspaces are
their own, so that replays run beside each other and beside other calls."""
import pytest
import torch

from paper_2607_18582_amd import Mure

pytestmark = pytest.mark.gpu

LENGTHS, D, N = [1500, 20, 2600, 513], 512, 16


@pytest.fixture()
def own():
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        m = Mure(device=0)
    yield m, side
    torch.cuda.synchronize()
    m.close()


def inputs(seed, mutants=1):
    g = torch.Generator().manual_seed(seed)
    T = sum(LENGTHS)
    rows = lambda c: torch.randn(mutants, T, c, generator=g).cuda()  # noqa: E731
    A = -torch.arange(1, N + 1) * torch.exp(torch.randn(D, N, generator=g) * 0.1)
    return rows(D), rows(D) - 4, A.cuda(), rows(N), rows(N)


def capture(stream, call):
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        out = call()
    return graph, out


def test_a_capture_needs_no_call_before_it(own):
    print("[graphs] first", flush=True)
    m, side = own
    p = inputs(0)
    seqs = m.sequences(LENGTHS)
    torch.cuda.synchronize()
    graph, (y, last) = capture(side, lambda: seqs.scan(*p))
    with torch.cuda.stream(side):
        more = seqs.scan(*(v if v is p[2] else v.expand(3, *v.shape[1:]) + 0 for v in p))     # a larger workspace, made directly
        expected = seqs.scan(*p)
        side.synchronize()
        for i in range(4):
            y.zero_()
            graph.replay()
            side.synchronize()
            assert torch.equal(y, expected[0]) and torch.equal(last, expected[1]), i
            again = seqs.scan(*p)
            side.synchronize()
            assert torch.equal(again[0], expected[0]) and torch.equal(more[0][2], expected[0][0]), i


def test_graphs_beside_each_other(own):
    print("[graphs] beside", flush=True)
    m, side = own
    ps = [inputs(1), inputs(2, 2), inputs(3)]
    seqs = m.sequences(LENGTHS)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        expected = [seqs.scan(*p) for p in ps]
        side.synchronize()
    # the second graph has two scans, which share a workspace and follow each other
    first, out1 = capture(side, lambda: (seqs.scan(*ps[0]),))
    second, out2 = capture(side, lambda: (seqs.scan(*ps[1]), seqs.scan(*ps[2])))
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    for i in range(20):
        for t in [t for pair in out1 + out2 for t in pair]:
            t.zero_()
        torch.cuda.synchronize()
        with torch.cuda.stream(a):
            first.replay()
        with torch.cuda.stream(b):
            second.replay()
        with torch.cuda.stream(side):
            direct = seqs.scan(*ps[2])
        torch.cuda.synchronize()
        for got, e in zip(out1 + out2 + (direct,), expected + [expected[2]]):
            assert torch.equal(got[0], e[0]) and torch.equal(got[1], e[1]), i


def test_a_batch_closed_during_a_capture(own):
    """A batch that is closed, or found by the garbage collector, while its context's stream is captured."""
    print("[graphs] close", flush=True)
    m, side = own
    x, taps = torch.ones(604, 16, device="cuda"), torch.ones(16, 4, device="cuda")
    seqs, other = m.sequences([600, 4]), m.sequences([5000, 5])
    with torch.cuda.stream(side):
        many = torch.randn(5005, 512, device="cuda")
        expected = other.conv(many, torch.ones(512, 4, device="cuda"))[0]
        side.synchronize()
        taken = other.conv(many, torch.ones(512, 4, device="cuda"))[0]      # still running when the batch is closed

    def call():
        y, _ = seqs.conv(x, taps)
        other.close()
        return seqs.conv(y, taps)

    graph, (y, _) = capture(side, call)
    torch.cuda.synchronize()
    assert torch.equal(taken, expected)
    for i in range(3):
        y.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert float(y[3, 0]) == 1 + 2 + 3 + 4 and float(y[599, 5]) == 16, i
