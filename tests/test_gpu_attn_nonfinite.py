"""Attention where weights are too small for float32 or values are not finite:
what a value does to a result depends on its weight in the formula, not on the
tile, wave or part that holds its key."""
import pytest
import torch

import attn_reference as R
from paper_2607_18582_amd import Mure
from test_gpu_attn import TYPES, cuda, normal, say

pytestmark = pytest.mark.gpu

INF, NAN = float("inf"), float("nan")

# lengths and past of one sequence (None: no cache): waves on their own, runs; over a cache single tokens, few, runs over parts
# and runs over all keys
SHAPES = [(40, None), (96, None), (300, None), (1, 2600), (7, 1500), (1, 300), (40, 2200), (530, 100)]


@pytest.fixture(scope="module")
def mure():
    m = Mure(device=0)
    yield m
    m.close()


def steep(seed, count, past, dim, dtype, peaks):
    """Queries and keys whose scores are 0, but `peaks`' (key: score; multiples of 16), and values."""
    total = (past or 0) + count
    g = torch.Generator().manual_seed(seed)
    q, k = torch.zeros(1, count, 2 * dim, dtype=dtype), torch.zeros(1, total, dim, dtype=dtype)
    q[..., 0] = q[..., dim] = 16
    for j, s in peaks.items():
        k[0, j, 0] = s / 16
    return q, k, normal(g, 1, total, dim, dtype=dtype)


def check(mure, q, k, v, count, past, dim, what, bound_from=None, **how):
    """bound_from: keys and values whose results have the bounds that are meant."""
    at = past or 0
    cache, p = None, None
    if past is not None:
        cache, p = [], torch.tensor([past], dtype=torch.int32)
        for t in (k, v):
            cache.append(torch.full((1, 1, past + count + 3, dim), NAN, dtype=q.dtype))
            cache[-1][0, 0, :past] = t[0, :past]
    expected = R.attend(q, k[:, at:], v[:, at:], [count], dim, scale=1.0, cache=cache, past=p, **how)[0]
    if bound_from:
        held = None if past is None else [t[:, None].clone() for t in bound_from]
        bound = R.attend(q, *(t[:, at:] for t in bound_from), [count], dim, scale=1.0, cache=held, past=p, **how)[0][1]
        expected = expected[0], bound
    out = mure.sequences([count]).attend(*cuda(q, k[:, at:], v[:, at:]), head_dim=dim, scale=1.0, cache=cache and cuda(*cache), past=cuda(p)[0], **how)
    R.close(out, expected, what)


def places(total):
    """Keys at the ends of blocks, tiles, waves' shares and parts, and the middle."""
    return sorted({j for j in (0, 1, 15, 16, 31, 32, 63, 64, 127, 128, 511, 512, 1023, 1024, 2047, total // 2, total - 2, total - 1) if 0 <= j < total})


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("count,past", SHAPES)
@pytest.mark.parametrize("dim,how", [(64, {}), (64, {"causal": False}), (66, {}), (17, {"window": 70}), (200, {})])
def test_infinite_values_of_small_weight(mure, dtype, count, past, dim, how):
    """Weights of e^-200 and e^-400 times infinity are infinite, wherever keys, peaks and values lie."""
    say(f"[small weights, inf] {dtype} {count} {past} dim={dim} {how}")
    total = (past or 0) + count
    for n, peak in enumerate((total - 1, 0, total // 2, min(40, total - 1))):
        q, k, v = steep(60 + n, count, past, dim, TYPES[dtype], {total // 3: 192, peak: 400})
        for c, j in enumerate(places(total)):
            v[0, j, c % (dim - 3)] = (INF, -INF)[c % 2]
        v[0, total // 4, dim - 3] = NAN
        v[0, total // 5, dim - 2], v[0, total - 1 - total // 5, dim - 2] = INF, -INF
        check(mure, q, k, v, count, past, dim, f"peak at {peak}", **how)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("count,past", SHAPES)
@pytest.mark.parametrize("dim,how", [(64, {}), (66, {"causal": False}), (128, {"window": 40}), (200, {})])
def test_infinite_values_of_no_weight(mure, dtype, count, past, dim, how):
    """A score of -inf is a weight of 0: a finite value counts for nothing, and 0 times infinity is NaN."""
    say(f"[no weight, inf] {dtype} {count} {past} dim={dim} {how}")
    total = (past or 0) + count
    q, k, v = steep(80, count, past, dim, TYPES[dtype], {total // 3: 192})
    plain = k.clone(), v.clone()               # the same finite results, by weights of e^-480
    for c, j in enumerate(places(total)):
        if c % 2 and j != total // 3:
            k[0, j, 0], plain[0][0, j, 0], plain[1][0, j] = -INF, -30, 0
        v[0, j, c] = INF
    check(mure, q, k, v, count, past, dim, "values beside keys of -inf", plain, **how)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("count,past", SHAPES)
@pytest.mark.parametrize("dim", [64, 200])
def test_huge_values_of_small_weight(mure, dtype, count, past, dim):
    """1e38 times e^-200 and less is nothing beside the peak's own values."""
    say(f"[small weights, huge] {dtype} {count} {past} dim={dim}")
    total = (past or 0) + count
    for n, peak in enumerate((total - 1, total // 2, min(40, total - 1))):
        q, k, v = steep(70 + n, count, past, dim, TYPES[dtype], {peak: 400})
        for c, j in enumerate(places(total)):
            if j != peak:
                v[0, j, c % dim] = (1e38, -1e38)[c % 2]
        check(mure, q, k, v, count, past, dim, f"peak at {peak}")
