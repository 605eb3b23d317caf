"""The operators of an attention block, for measurement.

Between plain projections and norms, a block of such a sequence model is

* the norms of queries and keys for each head and the rotation of their pairs
  of channels by the token's position (or several: time, height, width);
* attention of every token over its sequence: a softmax of scaled products of
  queries and keys weighs the values; several heads of queries share one of
  keys and values.  A cache holds the keys and values of earlier tokens;
* the gated feed-forward layer: two projections, one of them through an
  activation, and the product of both.

As everywhere in this repository one call evaluates many mutants of a network
over the same test set: a tensor has a leading mutant axis, or none when all
mutants share it (activations of the original model, unmutated parameters).
Sequences are packed one after the other, of any lengths.

Every case names one operator ("op"), its types and sizes.  The lengths of the
sequences come from the case alone, the values from the seed.  ``run`` makes
one pass: in plain torch operations in float32, or (``own``) through the
library's calls.  Values have the scale that a trained block sees.
"""
import random

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
EPS = 1e-6


# ---------------------------------------------------------------- the cases

def _named(name, **case):
    return case if name is None else {"name": name, **case}


def _rotate(name, dtype, seqs, shortest, longest, heads, kv_heads, head_dim, rotated, norm="rms", interleaved=False,
            axes=1, past=False, mutants=1):
    """rotated: channels of a head that take part.  past: positions count on from an earlier call's."""
    return _named(name, op="rotate", dtype=dtype, mutants=mutants, seqs=seqs, shortest=shortest, longest=longest,
                  heads=heads, kv_heads=kv_heads, head_dim=head_dim, rotated=rotated, norm=norm, interleaved=interleaved,
                  axes=axes, past=past)


def _attend(name, dtype, seqs, shortest, longest, heads, kv_heads, head_dim, causal=True, window=0, held=(0, 0),
            mutants=1, shared=False):
    """held: the fewest and the most tokens that a sequence's cache holds (no cache: 0).  shared: keys and values are
    the original model's."""
    return _named(name, op="attend", dtype=dtype, mutants=mutants, seqs=seqs, shortest=shortest, longest=longest,
                  heads=heads, kv_heads=kv_heads, head_dim=head_dim, causal=causal, window=window, held_least=held[0],
                  held_most=held[1], shared=shared)


def _gated(name, dtype, rows, inner, outer, activation="silu", bias=False, mutants=1, shared=False):
    """shared: the rows are the original model's and the weights mutated; otherwise the weights are the original's."""
    return _named(name, op="gated", dtype=dtype, mutants=mutants, rows=rows, inner=inner, outer=outer,
                  activation=activation, bias=bias, shared=shared)


def listed():
    return [
        # a decoding step: 64 sequences get one token each, at the positions after their caches
        _rotate("rotate, a token each", "bf16", 64, 1, 1, 16, 4, 128, 128, past=True),
        # a layer after the mutated one, over sequences of the RNN workload's lengths: every mutant has activations of
        # its own; neighbouring channels make the pairs, half of them turn
        _rotate("rotate, mutants' reviews", "f32", 250, 20, 80, 4, 2, 32, 16, norm="layer", interleaved=True, mutants=16),
        # patches of a video: time, height and width each turn a third of the pairs
        _rotate("rotate, video", "bf16", 1, 65536, 65536, 16, 4, 96, 96, axes=3),
        # the same decoding step: one token each over caches of very different lengths
        _attend("attend, a token each", "bf16", 64, 1, 1, 16, 4, 128, held=(500, 8000)),
        # one sequence with a long cache: little but the cache to work on side by side
        _attend("attend, one long cache", "bf16", 1, 1, 1, 32, 8, 128, held=(100001, 100001)),
        # the first mutated layer is a projection of queries: the classifier's tokens see each other both ways, keys
        # and values are the memoized ones
        _attend("attend, mutated queries", "f32", 250, 20, 80, 4, 4, 32, causal=False, mutants=16, shared=True),
        # prompts of very different lengths in one batch, a head size that fits no power of two
        _attend("attend, ragged prompts", "bf16", 12, 17, 4000, 12, 4, 80),
        # one long document
        _attend("attend, long prompt", "bf16", 1, 16384, 16384, 16, 4, 128),
        # the same decoding step
        _gated("gated, a token each", "bf16", 64, 2048, 5632),
        # the first mutated layer is a gated one: 16 mutants' weights over the memoized rows, an odd number of neurons
        _gated("gated, mutated neurons", "f32", 12500, 128, 341, bias=True, mutants=16, shared=True),
        # widths that fit no vector
        _gated("gated, odd widths", "bf16", 5003, 1003, 2675, activation="gelu"),
        # the long document through a wide block
        _gated("gated, long prompt", "bf16", 16384, 4096, 11008),
    ]


def _log(rng, lo, hi):
    """A whole number between lo and hi, spread over their logarithm."""
    return max(lo, min(hi, round(lo * (hi / lo) ** rng.random())))


def draw(rng):
    op = rng.choice(["rotate", "attend", "attend", "gated"])
    dtype = rng.choice(["f32", "bf16"])
    mutants = rng.choice([1, 1, _log(rng, 2, 32)])
    if op == "gated":
        inner, outer = _log(rng, 64, 4096), _log(rng, 64, 11008)
        # products and results of a drawn case: products of float32 cost several times as much
        most = min((1 << (38 if dtype == "bf16" else 35)) // (inner * outer * mutants), (1 << 27) // (max(inner, outer) * mutants))
        return _gated(None, dtype, _log(rng, 1, max(1, min(16384, most))), inner, outer, activation=rng.choice(["silu", "gelu"]),
                      bias=rng.random() < 0.5, mutants=mutants, shared=rng.random() < 0.5 and inner * outer * mutants < 1 << 26)
    kv_heads = _log(rng, 1, 8)
    heads = kv_heads * rng.choice([1, 2, 3, 4, 8])
    head_dim = rng.choice([32, 64, 128, 128, 2 * _log(rng, 8, 128)])
    seqs = _log(rng, 1, 64)
    if op == "rotate":
        most = (1 << (27 if dtype == "bf16" else 26)) // (mutants * (heads + kv_heads) * head_dim)
        longest = _log(rng, 1, max(1, min(32768, most // seqs)))
        axes = rng.choice([1, 1, 3]) if head_dim >= 32 else 1
        rotated = rng.choice([head_dim, max(2, head_dim // 4 * 2)])
        return _rotate(None, dtype, seqs, _log(rng, 1, longest), longest, heads, kv_heads, head_dim, rotated,
                       norm=rng.choice(["rms", "rms", "layer", None]), interleaved=rng.random() < 0.3, axes=axes,
                       past=axes == 1 and rng.random() < 0.5, mutants=mutants)
    # scores of a drawn case, as the plain form lays them out; tokens of its sequences and of their caches
    scores = (1 << (32 if dtype == "bf16" else 30)) // (mutants * heads * seqs)
    elements = (1 << (27 if dtype == "bf16" else 26)) // (mutants * seqs * head_dim)
    tokens, kept = elements // heads, elements // kv_heads
    held = (0, 0)
    if rng.random() < 0.5:
        longest = rng.choice([1, 1, _log(rng, 2, 512)])
        longest = max(1, min(longest, int(scores ** 0.5), tokens))
        most = _log(rng, 1, max(1, min(131072, kept, scores // longest - longest)))
        held = (_log(rng, 1, most), most)
    else:
        longest = _log(rng, 1, max(1, min(16384, int(scores ** 0.5), tokens)))
    causal = rng.random() < 0.7
    return _attend(None, dtype, seqs, _log(rng, 1, longest), longest, heads, kv_heads, head_dim, causal=causal,
                   window=rng.choice([0, 0, 0, _log(rng, 1, 4096)]), held=held, mutants=mutants,
                   shared=held[1] == 0 and rng.random() < 0.3)


def _spread(n, lo, hi):
    """n whole numbers from lo to hi in even steps of their logarithm, in mixed order."""
    got = [round(lo * (hi / lo) ** (i / max(1, n - 1))) for i in range(n - 1)] + [hi]
    random.Random(n).shuffle(got)
    return got


def lengths(case):
    return _spread(case["seqs"], case["shortest"], case["longest"])


def held(case):
    """Tokens that each sequence's cache holds before the call."""
    return _spread(case["seqs"], case["held_least"], case["held_most"])[::-1] if case["held_most"] else [0] * case["seqs"]


def work(case):
    M, e = case["mutants"], 4 if case["dtype"] == "f32" else 2
    if case["op"] == "gated":
        R, K, N = case["rows"], case["inner"], case["outer"]
        own_rows, own_weights = (1, M) if case["shared"] else (M, 1)
        return {"bytes": e * (own_rows * R * K + own_weights * 2 * K * N + M * R * N) + (8 * own_weights * N if case["bias"] else 0),
                "flops": M * R * N * (4 * K + 8)}
    T, H, G, d = sum(lengths(case)), case["heads"], case["kv_heads"], case["head_dim"]
    if case["op"] == "rotate":
        n = M * T * (H + G) * d
        return {"bytes": 2 * n * e + (4 * T * case["axes"] if case["axes"] > 1 else 0) + 8 * d + 2 * case["rotated"], "flops": 9 * n}
    pairs = 0                                               # of a token and a key that it sees, per head
    W = case["window"] or 1 << 40
    for n, p in zip(lengths(case), held(case)):
        t = torch.arange(p, p + n)
        last = t + 1 if case["causal"] else torch.clamp(t + W, max=p + n)
        pairs += int((last - torch.clamp(t - W + 1, min=0)).sum())
    kept = sum(min(p, W + n) for n, p in zip(lengths(case), held(case)))
    kv = 1 if case["shared"] else M
    new = 2 * kv * T * G * d * e
    return {"bytes": 2 * M * T * H * d * e + new + (new + 2 * kv * kept * G * d * e if case["held_most"] else 0),
            "flops": M * H * pairs * (4 * d + 4)}


# ---------------------------------------------------------------- the inputs

def prepare(case, seed):
    device = torch.device("cuda")
    g = torch.Generator(device=device).manual_seed(seed)
    dt, M = TYPES[case["dtype"]], case["mutants"]

    def normal(*shape, dtype=torch.float32, mean=0.0, std=1.0):
        return (torch.randn(*shape, generator=g, device=device) * std + mean).to(dtype)

    s = {"case": case}
    if case["op"] == "gated":
        R, K, N = case["rows"], case["inner"], case["outer"]
        s["x"] = normal(R, K, dtype=dt) if case["shared"] else normal(M, R, K, dtype=dt)
        wide = (M,) if case["shared"] else ()
        s["gate"], s["up"] = normal(*wide, N, K, dtype=dt, std=K ** -0.5), normal(*wide, N, K, dtype=dt, std=K ** -0.5)
        s["gate_bias"], s["up_bias"] = (normal(*wide, N, std=0.1), normal(*wide, N, std=0.1)) if case["bias"] else (None, None)
        if own:
            s["library"] = _library()
        return s
    lens, n, H, G, d = lengths(case), case["seqs"], case["heads"], case["kv_heads"], case["head_dim"]
    T = sum(lens)
    # queries, keys and values side by side, as one projection leaves them
    kv_mutants = 1 if case.get("shared") else M
    if kv_mutants == M:
        rows = normal(M, T, (H + 2 * G) * d, dtype=dt)
        s["q"], s["k"], s["v"] = rows[..., :H * d], rows[..., H * d:(H + G) * d], rows[..., (H + G) * d:]
    else:
        rows = normal(T, 2 * G * d, dtype=dt)
        s["q"], s["k"], s["v"] = normal(M, T, H * d, dtype=dt), rows[:, :G * d], rows[:, G * d:]
    # the packed rows: each one's sequence and its position there, each sequence's first row and length
    count = torch.tensor(lens, device=device)
    s["seq"] = torch.repeat_interleave(torch.arange(n, device=device), count)
    s["start"], s["count"] = torch.cumsum(count, 0) - count, count
    s["at"] = torch.arange(T, device=device) - s["start"][s["seq"]]
    s["past"] = s["positions"] = s["cache"] = None
    if case["op"] == "rotate":
        pairs, A = case["rotated"] // 2, case["axes"]
        s["frequencies"] = (10000.0 ** (-torch.arange(pairs, device=device, dtype=torch.float64) / pairs)).float()
        s["q_weight"], s["k_weight"] = (normal(d, mean=1.0, std=0.1), normal(d, mean=1.0, std=0.1)) if case["norm"] else (None, None)
        s["sections"] = None
        if A > 1:                                           # frames of 64 x 64 patches
            s["positions"] = torch.stack((s["at"] // 4096, s["at"] // 64 % 64, s["at"] % 64)).to(torch.int32)
            s["sections"] = [pairs - 2 * (pairs // 3), pairs // 3, pairs // 3]
        if case["past"]:
            s["past"] = torch.randint(0, 131072, (n,), generator=g, device=device).to(torch.int32)
    elif case["held_most"]:
        s["past"] = torch.tensor(held(case), device=device, dtype=torch.int32)
        capacity = max(a + b for a, b in zip(lens, held(case))) + 5
        s["cache"] = tuple(normal(M, n, capacity, G * d, dtype=dt) for _ in range(2))
    if own:                                                 # the library's form of the same: a handle made of the lengths
        s["sequences"] = _library().sequences(lens)
    return s


def _library():
    from paper_2607_18582_amd import Mure
    return Mure(device=torch.cuda.current_device())


# ---------------------------------------------------------------- one pass

def run(s):
    case = s["case"]
    if not own:
        return {"rotate": _plain_rotate, "attend": _plain_attend, "gated": _plain_gated}[case["op"]](s)
    if case["op"] == "gated":
        return s["library"].gated(s["x"], s["gate"], s["up"], gate_bias=s["gate_bias"], up_bias=s["up_bias"],
                                  activation=case["activation"])
    if case["op"] == "rotate":
        return s["sequences"].rotate(s["q"], s["k"], s["frequencies"], head_dim=case["head_dim"], norm=case["norm"],
                                     q_weight=s["q_weight"], k_weight=s["k_weight"], eps=EPS, past=s["past"],
                                     positions=s["positions"], sections=s["sections"], interleaved=case["interleaved"])
    out = s["sequences"].attend(s["q"], s["k"], s["v"], head_dim=case["head_dim"], causal=case["causal"],
                                window=case["window"] or None, cache=s["cache"], past=s["past"])
    return out if s["cache"] is None else (out, *s["cache"])


def _plain_rotate(s):
    case = s["case"]
    d, R = case["head_dim"], case["rotated"]
    if s["positions"] is None:
        at = s["at"] if s["past"] is None else s["at"] + s["past"][s["seq"]]
        at = at[:, None]
    else:
        at = torch.cat([p[:, None].expand(-1, c) for p, c in zip(s["positions"], s["sections"])], 1)
    angle = at.double() * s["frequencies"].double()         # in 64 bits: far positions
    cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]

    def one(x, weight):
        v = x.float().unflatten(-1, (-1, d))
        if case["norm"] == "layer":
            v = v - v.mean(-1, keepdim=True)
        if case["norm"]:
            v = v * torch.rsqrt((v * v).mean(-1, keepdim=True) + EPS) * weight
        turned = v[..., :R]
        if case["interleaved"]:
            a, b = turned[..., 0::2], turned[..., 1::2]
            turned = torch.stack((a * cos - b * sin, a * sin + b * cos), -1).flatten(-2)
        else:
            a, b = turned[..., :R // 2], turned[..., R // 2:]
            turned = torch.cat((a * cos - b * sin, a * sin + b * cos), -1)
        return torch.cat((turned, v[..., R:]), -1).flatten(-2).to(x.dtype)

    return one(s["q"], s["q_weight"]), one(s["k"], s["k_weight"])


def _plain_attend(s):
    """All sequences side by side, padded to the longest."""
    case = s["case"]
    H, G, d, W = case["heads"], case["kv_heads"], case["head_dim"], case["window"]
    M, n, L, device = case["mutants"], case["seqs"], case["longest"], s["q"].device
    steps = torch.arange(L, device=device)
    rows = (s["start"][:, None] + steps).clamp(max=s["seq"].numel() - 1)

    def padded(x, heads):                                   # [.., n, heads, L, d]
        return x.float()[..., rows, :].unflatten(-1, (heads, d)).transpose(-3, -2)

    at = steps.expand(n, L)
    if s["cache"] is None:
        k, v = padded(s["k"], G), padded(s["v"], G)
        key_at, there = at, steps < s["count"][:, None]
    else:
        past = s["past"].long()
        for held_rows, new in zip(s["cache"], (s["k"], s["v"])):
            held_rows[:, s["seq"], past[s["seq"]] + s["at"]] = new
        k, v = (c.float().unflatten(-1, (G, d)).transpose(-3, -2) for c in s["cache"])
        at = at + past[:, None]
        key_at = torch.arange(k.size(-2), device=device).expand(n, -1)
        there = key_at < (past + s["count"])[:, None]
    sees = there[:, None, :].expand(n, L, -1)
    if case["causal"]:
        sees = sees & (key_at[:, None, :] <= at[:, :, None])
    if W:
        sees = sees & ((key_at[:, None, :] - at[:, :, None]).abs() < W)
    q = padded(s["q"], H).unflatten(-3, (G, H // G)).flatten(-3, -2) * d ** -0.5    # [M, n, G, heads of a group x L, d]
    scores = torch.matmul(q, k.transpose(-2, -1).contiguous())
    scores = scores.view(M, n, G, H // G, L, -1).masked_fill_(~sees[:, None, None], float("-inf"))
    scores = scores.sub_(scores.amax(-1, keepdim=True).clamp_(min=-1e30)).exp_()
    total = scores.sum(-1, keepdim=True)
    out = torch.matmul(scores.flatten(-3, -2), v.contiguous()).view(M, n, H, L, d) / total.flatten(2, 3)
    out = out.transpose(-3, -2)[:, s["seq"], s["at"]].flatten(-2).to(s["q"].dtype)
    return out if s["cache"] is None else (out, *s["cache"])


def _plain_gated(s):
    a, b = (torch.matmul(s["x"].float(), s[w].float().transpose(-2, -1)) for w in ("gate", "up"))
    if s["gate_bias"] is not None:
        a, b = a + s["gate_bias"][..., None, :], b + s["up_bias"][..., None, :]
    if s["case"]["activation"] == "silu":
        a = a * torch.sigmoid(a)
    else:
        a = 0.5 * a * (1 + torch.erf(a * 0.5 ** 0.5))
    return (a * b).to(s["x"].dtype)


# ---------------------------------------------------------------- in 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    return {"rotate": _exact_rotate, "attend": _exact_attend, "gated": _exact_gated}[case["op"]](s)


def _exact_rotate(s):
    """Pairs as complex numbers, one head at a time."""
    case = s["case"]
    d, R = case["head_dim"], case["rotated"]
    if s["sections"] is None:
        position = s["at"].double()
        if s["past"] is not None:
            position = position + s["past"].double()[s["seq"]]
        angle = torch.outer(position, s["frequencies"].double())
    else:
        parts = s["frequencies"].double().split(s["sections"])
        angle = torch.cat([torch.outer(p.double(), f) for p, f in zip(s["positions"], parts)], 1)
    turn = torch.complex(torch.cos(angle), torch.sin(angle))
    outs = []
    for x, weight in ((s["q"], s["q_weight"]), (s["k"], s["k_weight"])):
        y = torch.empty(x.shape, dtype=torch.float64, device=x.device)
        for h in range(x.size(-1) // d):
            v = x[..., h * d:(h + 1) * d].double()
            if case["norm"] == "layer":
                v = v - v.sum(-1, keepdim=True) / d
            if case["norm"]:
                v = v / torch.sqrt(torch.square(v).sum(-1, keepdim=True) / d + EPS) * weight.double()
            first, second = (slice(0, R, 2), slice(1, R, 2)) if case["interleaved"] else (slice(0, R // 2), slice(R // 2, R))
            z = torch.complex(v[..., first].contiguous(), v[..., second].contiguous()) * turn
            v[..., first], v[..., second] = z.real, z.imag
            y[..., h * d:(h + 1) * d] = v
        outs.append(y)
    return tuple(outs)


def _exact_attend(s):
    """Sequence by sequence and head by head, some tokens at a time."""
    case = s["case"]
    H, G, d, M = case["heads"], case["kv_heads"], case["head_dim"], case["mutants"]
    device, row = s["q"].device, 0
    y = torch.empty(M, s["q"].size(-2), H * d, dtype=torch.float64, device=device)
    caches = None if s["cache"] is None else [c.double() for c in s["cache"]]
    for i, (count, p) in enumerate(zip(lengths(case), held(case))):
        rows = slice(row, row + count)
        keys, values = (x[..., rows, :].double().expand(M, -1, -1) for x in (s["k"], s["v"]))
        if caches is not None:
            for c, new in zip(caches, (keys, values)):
                c[:, i, p:p + count] = new
            keys, values = (c[:, i, :p + count] for c in caches)
        block = max(1, min(count, (1 << 27) // (M * (p + count))))
        for h in range(H):
            kv = slice(h // (H // G) * d, (h // (H // G) + 1) * d)
            for t0 in range(0, count, block):
                t1 = min(count, t0 + block)
                at = torch.arange(p + t0, p + t1, device=device)[:, None]
                # keys behind the last one that the block sees are left out
                last = p + t1 if case["causal"] else p + count
                j = torch.arange(last, device=device)
                hidden = torch.zeros(t1 - t0, last, dtype=torch.bool, device=device)
                if case["causal"]:
                    hidden |= j > at
                if case["window"]:
                    hidden |= (j - at).abs() >= case["window"]
                scores = torch.matmul(s["q"][:, row + t0:row + t1, h * d:(h + 1) * d].double(),
                                      keys[:, :last, kv].transpose(1, 2).contiguous()) / d ** 0.5
                weights = torch.softmax(scores.masked_fill_(hidden, float("-inf")), -1)
                y[:, row + t0:row + t1, h * d:(h + 1) * d] = torch.matmul(weights, values[:, :last, kv].contiguous())
        row += count
    return y if caches is None else (y, *caches)


def _exact_gated(s):
    x = s["x"].double()
    weights = [s[w].double() for w in ("gate", "up")]
    shape = (s["case"]["mutants"], s["case"]["rows"], s["case"]["outer"])
    y = torch.empty(shape, dtype=torch.float64, device=x.device)
    for m in range(shape[0]):
        one = x if x.dim() == 2 else x[m]
        a, b = (torch.mm(one, (w if w.dim() == 2 else w[m]).T) for w in weights)
        if s["gate_bias"] is not None:
            gate_bias, up_bias = (v.double() if v.dim() == 1 else v[m].double() for v in (s["gate_bias"], s["up_bias"]))
            a, b = a + gate_bias, b + up_bias
        if s["case"]["activation"] == "silu":
            a = a / (1 + torch.exp(-a))
        else:
            a = a * torch.special.ndtr(a)
        y[m] = a * b
    return y
