"""The example of memoized mutation testing of an attention classifier: the
logits of memoized and exhaustive evaluation are equal bit for bit, streaming
token by token gives what the whole sequences give, and the logits are those
of the definitions in float64."""
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
import attn_mutants as E  # noqa: E402
import attn_reference as R  # noqa: E402
from paper_2607_18582_amd import Mure  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def mure():
    m = Mure(device=0)
    yield m
    m.close()


def reference_logits(model, tokens, lengths, replaced=None):
    """In float64 on the CPU, from the operators' definitions."""
    cpu = lambda t: t.double().cpu()  # noqa: E731
    h = cpu(model.embedding)[tokens.cpu()]
    norm = lambda v, w: v * torch.rsqrt((v * v).mean(-1, keepdim=True) + 1e-5) * cpu(w)  # noqa: E731
    for i, b in enumerate(model.blocks):
        if replaced and replaced[0] == i:
            b = dict(b, **replaced[2])
        q, k, v = (norm(h, b["norm"]) @ cpu(b["qkv"])).split([E.HEADS * E.DIM, E.GROUPS * E.DIM, E.GROUPS * E.DIM], -1)
        q, k = (R.rotate(t[None], cpu(model.frequencies)[None], lengths, E.DIM, "rms", cpu(b[w])[None])[0]
                for t, w in ((q, "q_weight"), (k, "k_weight")))
        y = attention(q[0], k[0], v, lengths)
        h = h + y @ cpu(b["out"])
        x = norm(h, b["middle"])
        h = h + (torch.nn.functional.silu(x @ cpu(b["gate"]).T) * (x @ cpu(b["up"]).T)) @ cpu(b["down"])
    last = torch.cumsum(torch.tensor(lengths), 0) - 1
    return (norm(h, model.last_norm) @ cpu(model.head))[last]


def attention(q, k, v, lengths):
    out, row = torch.zeros_like(q), 0
    for n in lengths:
        s = slice(row, row + n)
        for h in range(E.HEADS):
            a, g = slice(h * E.DIM, (h + 1) * E.DIM), h // (E.HEADS // E.GROUPS)
            b = slice(g * E.DIM, (g + 1) * E.DIM)
            w = (q[s, a] @ k[s, b].T * E.DIM ** -0.5).masked_fill(torch.ones(n, n).triu(1).bool(), float("-inf"))
            out[s, a] = w.softmax(-1) @ v[s, b]
        row += n
    return out


def test_memoized_is_exhaustive_and_right(mure):
    print("[example] memoized against exhaustive", flush=True)
    model = E.make_model(blocks=2, width=64, inner=96, vocab=50, classes=5)
    lengths = [12, 1, 30, 7, 22, 150]
    tokens = torch.randint(0, 50, (sum(lengths),), generator=torch.Generator().manual_seed(3)).cuda()
    mutants = E.make_mutants(model, 10)
    ev = E.Evaluation(mure, model, lengths)
    original, logits = E.memoized(ev, tokens, mutants)
    assert torch.equal(logits, E.exhaustive(ev, tokens, mutants))
    assert len({(b, s) for b, s, _ in mutants}) == 4
    # float32 through two blocks, each five products of at most 128 terms and a softmax whose exponents (up to about 20)
    # carry their own rounding: 2 * (5 * 128 + 20 * 32) units of the largest logit
    most = 2560 * R.U * float(original.abs().max())
    assert float((original.cpu() - reference_logits(model, tokens, lengths)).abs().max()) <= most
    for i in (0, 3, 5, 8):
        expected = reference_logits(model, tokens, lengths, mutants[i])
        assert float((logits[i].cpu() - expected).abs().max()) <= most, i
        assert not torch.equal(logits[i], original)
    kills, (num, den) = E.score(original, logits)
    assert kills.shape == (10, 6) and 0 <= num <= den


def test_streaming_is_the_whole(mure):
    print("[example] streaming", flush=True)
    model = E.make_model(blocks=2, width=64, inner=96, vocab=50, classes=5, seed=4)
    lengths = [5, 1, 40]
    g = torch.Generator().manual_seed(5)
    prompts, more = torch.randint(0, 50, (46,), generator=g).cuda(), torch.randint(0, 50, (3, 3), generator=g).cuda()
    mutants = E.make_mutants(model, 6)
    found = E.stream(mure, model, mutants, prompts, lengths, more)
    start = [0, 5, 6]
    for step, (original, logits) in enumerate(found):
        parts = [torch.cat((prompts[s:s + n], more[:step, i])) for i, (s, n) in enumerate(zip(start, lengths))]
        whole = E.Evaluation(mure, model, [n + step for n in lengths])
        o, l = E.memoized(whole, torch.cat(parts), mutants)
        # both within the bound above of the same definitions
        most = 2 * 2560 * R.U * float(o.abs().max())
        assert float((original - o).abs().max()) <= most and float((logits - l).abs().max()) <= most, step
