"""Attention over caches whose parts of keys take more workspace than a call
has, or whose blocks are more than a launch has: in several rounds, over
sequences, mutants and heads, each with the bits of a call of its own."""
import pytest
import torch

from paper_2607_18582_amd import Mure
from test_gpu_attn import TYPES, say

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def mure():
    m = Mure(device=0)
    yield m
    m.close()


def rand(g, *shape, dtype=torch.float32):
    return torch.randn(*shape, generator=g, device="cuda").to(dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_single_tokens_in_three_rounds(mure, dtype):
    """600 sequences of one token: parts of 256 of them fit the workspace, and such a batch has no list of items."""
    say(f"[rounds, single tokens] {dtype}")
    M, H, dim, rows, n, dt = 64, 64, 2, 32768, 600, TYPES[dtype]
    g = torch.Generator(device="cuda").manual_seed(50)
    q = rand(g, M, n, H * dim, dtype=dt)
    k, v = (rand(g, n, dim, dtype=dt) for _ in range(2))
    cache = [rand(g, n, rows, dim, dtype=dt) for _ in range(2)]
    past = (torch.arange(n, device="cuda") * 977 % 5000).to(torch.int32)
    past[[0, 255, 256, 511, 512, 599]] = torch.tensor([0, rows - 1, 511, 20000, 512, 30000], dtype=torch.int32, device="cuda")
    alone = [c.clone() for c in cache]
    out = torch.full_like(q, 77.0)
    mure.sequences([1] * n).attend(q, k, v, head_dim=dim, cache=cache, past=past, out=out)
    one = mure.sequences([1])
    wrong = []
    for i in range(n):
        at = slice(i, i + 1)
        expected = one.attend(q[:, at], k[at], v[at], head_dim=dim, cache=[c[at] for c in alone], past=past[at])
        if not torch.equal(out[:, at], expected):
            wrong.append(i)
    assert not wrong
    assert all(torch.equal(c, a) for c, a in zip(cache, alone))
    assert all(torch.equal(c[torch.arange(n), past.long()], new) for c, new in zip(cache, (k, v)))


def free_bytes():
    torch.cuda.synchronize()
    return torch.cuda.mem_get_info()[0]


@pytest.mark.parametrize("lengths,M,H,G,dim,rows", [
    ([130], 200, 16, 2, 8, 131072),            # 2.1 GB of parts: mutants in rounds
    ([130], 1, 1024, 2, 4, 400000),            # 0.6 GB a group of heads: groups in rounds
    ([130], 1, 1024, 1, 4, 400000),            # ... which are one: heads in rounds
    ([16], 1, 1024, 1, 64, 300000)])           # the same of a short sequence, tokens and heads in one unit of rows
def test_one_sequence_in_several_rounds(lengths, M, H, G, dim, rows):
    """The workspace stays within 1 GiB where one sequence's parts take more."""
    say(f"[rounds, one sequence] {lengths} M={M} H={H} G={G} dim={dim} rows={rows}")
    mure = Mure(device=0)
    g = torch.Generator(device="cuda").manual_seed(51)
    n, past = lengths[0], torch.tensor([2500], dtype=torch.int32, device="cuda")
    q = rand(g, M, n, H * dim, dtype=torch.bfloat16)
    k, v = (rand(g, n, G * dim, dtype=torch.bfloat16) for _ in range(2))
    cache = [rand(g, 1, rows, G * dim, dtype=torch.bfloat16) for _ in range(2)]
    before = [c.clone() for c in cache]
    out = torch.full_like(q, 77.0)
    seqs = mure.sequences(lengths)
    free = free_bytes()
    seqs.attend(q, k, v, head_dim=dim, cache=cache, past=past, out=out)
    assert free - free_bytes() <= (1 << 30) + (64 << 20)
    for c, b, new in zip(cache, before, (k, v)):
        b[0, 2500:2500 + n] = new
        assert torch.equal(c, b)
    # every mutant's heads alone
    for m in range(M):
        for h in {0, 1, H // 4, H // 2 - 1, H // 2, H - 2, H - 1}:
            at, kv = slice(h * dim, (h + 1) * dim), slice(h // (H // G) * dim, (h // (H // G) + 1) * dim)
            alone = seqs.attend(q[m, :, at], k[:, kv], v[:, kv], head_dim=dim, cache=[b[..., kv] for b in before], past=past)
            assert torch.equal(out[m, :, at], alone), (m, h)
    mure.close()


def test_a_workspace_of_the_rows_that_there_are():
    """A batch of single tokens beside one of 50, and of 17 tokens: parts of as many rows as their sequences have."""
    say("[rounds, rows]")
    mure = Mure(device=0)
    g = torch.Generator(device="cuda").manual_seed(52)
    H, dim, rows = 32, 64, 65536
    # bytes of 128 parts of 512 keys or 64 of 1024, 66 floats a part and head
    for lengths, need in (([1] * 40 + [50], 40 * 32 * 128 * 66 * 4 + 50 * 32 * 64 * 66 * 4), ([17] * 20, 20 * 17 * 32 * 64 * 66 * 4)):
        T, n = sum(lengths), len(lengths)
        q, k, v = rand(g, T, H * dim, dtype=torch.bfloat16), rand(g, T, dim, dtype=torch.bfloat16), rand(g, T, dim, dtype=torch.bfloat16)
        cache = [torch.zeros(n, rows, dim, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        past, out, seqs = torch.full((n,), 600, dtype=torch.int32, device="cuda"), torch.empty_like(q), mure.sequences(lengths)
        free = free_bytes()
        seqs.attend(q, k, v, head_dim=dim, cache=cache, past=past, out=out)
        assert free - free_bytes() <= need + (64 << 20), lengths
        del cache
    mure.close()


def test_more_blocks_than_a_launch(mure):
    """Many mutants of few tokens, without a cache and over a long one: as many mutants a launch as it has blocks for."""
    say("[rounds, blocks]")
    g = torch.Generator(device="cuda").manual_seed(53)
    M, H, dim = 65535, 4, 2
    lengths = [1, 3]
    q, k, v = (rand(g, M, 4, H * dim) for _ in range(3))
    out = mure.sequences(lengths).attend(q, k, v, head_dim=dim)
    for m in (0, 1, 30000, M - 1):
        assert torch.equal(out[m], mure.sequences(lengths).attend(q[m], k[m], v[m], head_dim=dim)), m
    lengths = [97]
    q, k, v = (rand(g, M, 97, w * dim, dtype=torch.bfloat16) for w in (257, 1, 1))
    out = mure.sequences(lengths).attend(q, k, v, head_dim=dim)
    for m in (0, 1, 30000, M - 1):
        assert torch.equal(out[m], mure.sequences(lengths).attend(q[m], k[m], v[m], head_dim=dim)), m
    del q, k, v, out
    M, H, G, rows = 128, 32, 8, 131072
    q, (k, v) = rand(g, M, 3, H * dim), (rand(g, 3, G * dim) for _ in range(2))
    cache = [rand(g, 3, rows, G * dim) for _ in range(2)]
    past = torch.tensor([rows - 1, 5, 40000], dtype=torch.int32, device="cuda")
    alone = [c.clone() for c in cache]
    out = mure.sequences([1, 1, 1]).attend(q, k, v, head_dim=dim, cache=cache, past=past)
    for m in (0, 1, 77, M - 1):
        assert torch.equal(out[m], mure.sequences([1, 1, 1]).attend(q[m], k, v, head_dim=dim, cache=alone, past=past)), m
    assert all(torch.equal(c, a) for c, a in zip(cache, alone))


def test_rounds_in_a_graph():
    """Rounds over sequences and over heads, captured: every replay follows the pasts, beside direct calls."""
    say("[rounds, graph]")
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        mure = Mure(device=0)
    g = torch.Generator(device="cuda").manual_seed(54)
    for n, M, H, dim, rows in ((300, 64, 64, 2, 32768), (1, 2, 1024, 64, 300000)):
        lengths = [1] * n if n > 1 else [16]
        T = sum(lengths)
        q = rand(g, M, T, H * dim, dtype=torch.bfloat16)
        k, v = (rand(g, T, dim, dtype=torch.bfloat16) for _ in range(2))
        cache = [rand(g, n, rows, dim, dtype=torch.bfloat16) for _ in range(2)]
        start = (torch.arange(n, device="cuda") * 37 % 3000 + 100).to(torch.int32)
        past, held, seqs = start.clone(), [c.clone() for c in cache], mure.sequences(lengths)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            out = seqs.attend(q, k, v, head_dim=dim, cache=cache, past=past)
            past.add_(lengths[0])
        for i in range(4):
            graph.replay()
            torch.cuda.synchronize()
            with torch.cuda.stream(side):
                expected = seqs.attend(q, k, v, head_dim=dim, cache=held, past=start + i * lengths[0])
                side.synchronize()
            assert torch.equal(out, expected), (n, i)
            assert all(torch.equal(c, h) for c, h in zip(cache, held)), (n, i)
    torch.cuda.synchronize()
    del graph
    mure.close()
