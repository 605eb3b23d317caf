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
