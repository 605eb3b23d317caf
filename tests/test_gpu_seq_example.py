"""The example of memoized mutation testing of a state space classifier: the
logits of memoized and exhaustive evaluation are equal bit for bit, streaming
token by token gives what the whole sequences give, and the logits are those
of the definitions in float64."""
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
import seq_reference as R  # noqa: E402
import ssm_mutants as E  # noqa: E402
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
        xz = norm(h, b["norm"]) @ cpu(b["into"])
        channels = b["bias"].size(0)
        u = R.conv(xz[None, :, :channels], cpu(b["taps"])[None], cpu(b["bias"])[None], lengths, "silu")[0][0]
        low = u[0] @ cpu(b["select"])
        y = R.scan(u, (low[:, :E.RANK] @ cpu(b["dt"]))[None], cpu(b["A"])[None], low[None, :, E.RANK:E.RANK + E.STATES],
                   low[None, :, E.RANK + E.STATES:], lengths, cpu(b["skip"])[None], cpu(b["dt_bias"])[None],
                   xz[None, :, channels:])[0][0]
        h = h + y[0] @ cpu(b["out"])
    last = torch.cumsum(torch.tensor(lengths), 0) - 1
    return (norm(h, model.last_norm) @ cpu(model.head))[last]


def test_memoized_is_exhaustive_and_right(mure):
    print("[example] memoized against exhaustive", flush=True)
    model = E.make_model(blocks=2, width=64, channels=96, vocab=50, classes=5)
    lengths = [12, 1, 30, 7, 22]
    tokens = torch.randint(0, 50, (sum(lengths),), generator=torch.Generator().manual_seed(3)).cuda()
    mutants = E.make_mutants(model, 10)
    ev = E.Evaluation(mure, model, lengths)
    original, logits, _, _ = E.memoized(ev, tokens, mutants)
    assert torch.equal(logits, E.exhaustive(ev, tokens, mutants))
    assert len({(b, s) for b, s, _ in mutants}) == 4
    # float32 through two blocks of sums over at most 96 terms and 30 steps: a few hundred units of the largest logit
    most = 400 * R.U * float(original.abs().max())
    assert float((original.cpu() - reference_logits(model, tokens, lengths)).abs().max()) <= most
    for i in (0, 3, 5, 8):
        expected = reference_logits(model, tokens, lengths, mutants[i])
        assert float((logits[i].cpu() - expected).abs().max()) <= most, i
        assert not torch.equal(logits[i], original)
    kills, (num, den) = E.score(original, logits)
    assert kills.shape == (10, 5) and 0 <= num <= den


def test_streaming_is_the_whole(mure):
    print("[example] streaming", flush=True)
    model = E.make_model(blocks=2, width=64, channels=96, vocab=50, classes=5, seed=4)
    lengths = [5, 1, 9]
    g = torch.Generator().manual_seed(5)
    prompts, more = torch.randint(0, 50, (15,), generator=g).cuda(), torch.randint(0, 50, (3, 3), generator=g).cuda()
    mutants = E.make_mutants(model, 6)
    found = E.stream(mure, model, mutants, prompts, lengths, more)
    start = [0, 5, 6]
    for step, (original, logits) in enumerate(found):
        parts = [torch.cat((prompts[s:s + n], more[:step, i])) for i, (s, n) in enumerate(zip(start, lengths))]
        whole = E.Evaluation(mure, model, [n + step for n in lengths])
        o, l, _, _ = E.memoized(whole, torch.cat(parts), mutants)
        # the operators give the same bits either way; the projections' products have other shapes
        most = 100 * R.U * float(o.abs().max())
        assert float((original - o).abs().max()) <= most and float((logits - l).abs().max()) <= most, step
