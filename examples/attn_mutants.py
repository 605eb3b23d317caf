"""Memoized mutation testing of an attention classifier.

    python examples/attn_mutants.py [--mutants 24] [--sequences 200] [--blocks 2]

The network reads token sequences of different lengths: an embedding, blocks of
(projections to queries, keys and values, norm and rotation of every head,
causal attention with shared heads of keys and values, projection; gated layer,
projection) in a residual stream with norms, and a classifier on each
sequence's last token.  Weights are random and seeded.  A mutant changes a few
neurons of one block's gated layer, or a few heads' queries, by the operators
of the rest of the library: Gaussian noise on the incoming weights, their
negation, or zeros.

The original runs once and its activations are kept.  The mutants of one layer
(a cluster) then run together from that layer on: the memoized inputs are
shared by all of them, keys and values of the mutated block too, the mutated
parameters have a mutant axis, and so has everything after it.  A mutant kills
an input when its class differs from the original's.  The same mutants are
evaluated without memoization too, each from the tokens on: by the soundness
theorem (Section 4.1, Theorem 1) the outputs are the same, and they are
compared bit for bit.

``stream`` goes on token by token: every sequence gets one more token at a time,
over caches of the keys and values before it.  In the mutated block those are
the original's, and the mutants share one cache; behind it each has its own.

The projections are plain matrix products, one call for each mutant, so that
their shapes (and with them the library kernels that compute them) are the same
however many mutants are evaluated together.
"""
import argparse
import os
import sys
from types import SimpleNamespace

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2607_18582_amd import Mure  # noqa: E402

HEADS, GROUPS, DIM = 4, 2, 32
STAGES = ("attend", "gated")                    # the layers of a block that mutants change
MUTATED = {"attend": "q_weight", "gated": "gate"}


def make_model(blocks=2, width=128, inner=256, vocab=2000, classes=10, seed=0, device="cuda"):
    g = torch.Generator().manual_seed(seed)

    def normal(*shape, std=1.0, mean=0.0):
        return (torch.randn(*shape, generator=g) * std + mean).to(device)

    m = SimpleNamespace(embedding=normal(vocab, width), blocks=[], head=normal(width, classes, std=width ** -0.5),
                        last_norm=normal(width, mean=1.0, std=0.1), frequencies=(1000.0 ** (-torch.arange(DIM // 2) / (DIM // 2))).to(device))
    for _ in range(blocks):
        m.blocks.append(dict(
            norm=normal(width, mean=1.0, std=0.1), qkv=normal(width, (HEADS + 2 * GROUPS) * DIM, std=width ** -0.5),
            q_weight=normal(DIM, mean=2.0, std=0.5), k_weight=normal(DIM, mean=2.0, std=0.5), out=normal(HEADS * DIM, width, std=(HEADS * DIM) ** -0.5),
            middle=normal(width, mean=1.0, std=0.1), gate=normal(inner, width, std=width ** -0.5), up=normal(inner, width, std=width ** -0.5),
            down=normal(inner, width, std=inner ** -0.5)))
    return m


def make_mutants(model, count, seed=1):
    """(block, stage, the parameters it replaces) of each mutant."""
    g = torch.Generator().manual_seed(seed)
    mutants = []
    for i in range(count):
        block, stage = (i // 2) % len(model.blocks), STAGES[i % 2]
        w = model.blocks[block][MUTATED[stage]].clone()
        chosen = torch.randperm(w.size(0), generator=g)[:max(1, w.size(0) // 16)].to(w.device)
        op = i % 3
        if op == 0:                             # noise, of half the weights' size
            w[chosen] *= 1 + 0.5 * torch.randn(w[chosen].shape, generator=g).to(w.device)
        else:                                   # the pre-activation negated, or zero
            w[chosen] *= -1 if op == 1 else 0
        mutants.append((block, stage, {MUTATED[stage]: w}))
    return mutants


def project(x, w):
    return x @ w if x.dim() == 2 else torch.stack([one @ w for one in x])


def caches(model, lead, count, rows):
    """Empty caches of keys and values of one block, for `lead` mutants (() for the original)."""
    return tuple(torch.zeros(*lead, count, rows, GROUPS * DIM, device=model.head.device) for _ in range(2))


class Evaluation:
    """The network over a batch of sequences, from any layer of it on."""

    def __init__(self, mure, model, lengths):
        self.mure, self.model = mure, model
        self.sequences = mure.sequences(lengths)
        self.last = (torch.cumsum(torch.tensor(self.sequences.lengths), 0) - 1).to(model.head.device)

    def embed(self, tokens):
        """The inputs of the first block's attention."""
        h = self.model.embedding[tokens]
        b = self.model.blocks[0]
        _, x = self.mure.block_norm(h, before="rms", before_weight=b["norm"], residual_out=False)
        return {"residual": h, "qkv": project(x, b["qkv"])}

    def run(self, at, block=0, stage="attend", replaced=None, held=None, past=None, keep=None):
        """Logits from the inputs `at` of one block's stage on.  replaced: parameters of that
        block in place of the model's.  held: the caches of every block (None without them), past the tokens in
        them.  keep: receives the inputs of every (block, stage)."""
        for i in range(block, len(self.model.blocks)):
            b = dict(self.model.blocks[i], **(replaced if i == block and replaced else {}))
            if not (i == block and stage == "gated"):
                if keep is not None:
                    keep[i, "attend"] = at
                q, k, v = at["qkv"].split([HEADS * DIM, GROUPS * DIM, GROUPS * DIM], -1)
                q, _ = self.sequences.rotate(q, None, self.model.frequencies, head_dim=DIM, norm="rms", q_weight=b["q_weight"], past=past)
                k, _ = self.sequences.rotate(k, None, self.model.frequencies, head_dim=DIM, norm="rms", q_weight=b["k_weight"], past=past)
                y = self.sequences.attend(q, k, v, head_dim=DIM, cache=None if held is None else held[i], past=past)
                h, x = self.mure.block_norm(project(y, b["out"]), at["residual"], before="rms", before_weight=b["middle"])
                at = {"residual": h, "x": x}
            if keep is not None:
                keep[i, "gated"] = at
            y = self.mure.gated(at["x"], b["gate"], b["up"])
            last = i + 1 == len(self.model.blocks)
            weight = self.model.last_norm if last else self.model.blocks[i + 1]["norm"]
            h, x = self.mure.block_norm(project(y, b["down"]), at["residual"], before="rms", before_weight=weight)
            if last:
                return project(x[..., self.last, :].contiguous(), self.model.head)
            at = {"residual": h, "qkv": project(x, self.model.blocks[i + 1]["qkv"])}


def clusters(mutants):
    """Mutant ids by their mutated layer."""
    found = {}
    for i, (block, stage, _) in enumerate(mutants):
        found.setdefault((block, stage), []).append(i)
    return found


def stacked(mutants, ids):
    return {k: torch.stack([mutants[i][2][k] for i in ids]) for k in mutants[ids[0]][2]}


def memoized(ev, tokens, mutants, held=None, own=None, past=None):
    """(original's logits, every mutant's).  held: the original's caches; own: those of each cluster's mutants."""
    memo, logits = {}, [None] * len(mutants)
    original = ev.run(ev.embed(tokens), held=held, past=past, keep=memo)
    for (block, stage), ids in clusters(mutants).items():
        out = ev.run(memo[block, stage], block, stage, stacked(mutants, ids), None if own is None else own[block, stage], past)
        for i, one in zip(ids, out):
            logits[i] = one
    return original, torch.stack(logits)


def exhaustive(ev, tokens, mutants):
    """Every mutant's logits, each from the tokens on."""
    model, logits = ev.model, []
    for block, stage, own in mutants:
        ev.model = SimpleNamespace(**dict(vars(model), blocks=[dict(b, **own) if i == block else b for i, b in enumerate(model.blocks)]))
        logits.append(ev.run(ev.embed(tokens)))
    ev.model = model
    return torch.stack(logits)


def score(original, logits):
    """The kill matrix [mutants][sequences] and the mutation score as (killing labels, mutants x labels)."""
    label = original.argmax(-1)
    kills = logits.argmax(-1) != label
    labels = label.unique()
    killing = sum(int((kills & (label == k)).any(-1).sum()) for k in labels)
    return kills, (killing, len(logits) * len(labels))


def stream(mure, model, mutants, prompts, lengths, more):
    """Logits of the original and of every mutant after the prompts and each of the further tokens
    more [steps][sequences]: the prompts once, then one token for each sequence at a time, mutants of one layer
    together.  A mutated block's keys and values are the original's, so its mutants share one cache there."""
    n, blocks, rows = len(lengths), len(model.blocks), max(lengths) + len(more)
    held = [caches(model, (), n, rows) for _ in range(blocks)]
    own = {(block, stage): [caches(model, () if i == block else (len(ids),), n, rows) if i >= block else None for i in range(blocks)]
           for (block, stage), ids in clusters(mutants).items()}
    past = torch.zeros(n, dtype=torch.int32, device=prompts.device)
    found = [memoized(Evaluation(mure, model, lengths), prompts, mutants, held, own, past)]
    past += torch.tensor(lengths, dtype=torch.int32, device=past.device)
    step = Evaluation(mure, model, [1] * n)
    for tokens in more:
        found.append(memoized(step, tokens, mutants, held, own, past))
        past += 1
    return found


def main():
    p = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    p.add_argument("--mutants", type=int, default=24)
    p.add_argument("--sequences", type=int, default=200)
    p.add_argument("--blocks", type=int, default=2)
    a = p.parse_args()
    mure, model = Mure(device=0), make_model(a.blocks)
    g = torch.Generator().manual_seed(2)
    lengths = torch.randint(20, 81, (a.sequences,), generator=g).tolist()
    tokens = torch.randint(0, 2000, (sum(lengths),), generator=g).cuda()
    mutants = make_mutants(model, a.mutants)
    ev = Evaluation(mure, model, lengths)
    original, logits = memoized(ev, tokens, mutants)
    kills, (num, den) = score(original, logits)
    same = torch.equal(logits, exhaustive(ev, tokens, mutants))
    print(f"{a.mutants} mutants x {a.sequences} sequences: {int(kills.sum())} kills, mutation score {num}/{den} = {num / den:.3f}; "
          f"logits {'equal' if same else 'DIFFER from'} those without memoization, bit for bit")
    more = torch.randint(0, 2000, (3, a.sequences), generator=g).cuda()
    for i, (o, l) in enumerate(stream(mure, model, mutants, tokens, lengths, more)):
        print(f"after {i} more tokens: {int(score(o, l)[0].sum())} kills")
    return 0 if same else 1


if __name__ == "__main__":
    sys.exit(main())
