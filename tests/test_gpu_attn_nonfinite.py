"""Attention where weights are too small for float32 or values are not finite:
what a value does to a result depends on its weight in the formula, not on the
tile, wave or part that holds its key."""
import pytest
import torch

import attn_reference as R
from paper_2607_18582_amd import Mure
from test_gpu_attn import TYPES, cuda, held, normal, say

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


def check(mure, q, k, v, count, past, dim, what, scale=1.0, **how):
    if past is None:
        out = mure.sequences([count]).attend(*cuda(q, k, v), head_dim=dim, scale=scale, **how)
        expected = R.attend(q, k, v, [count], dim, scale=scale, **how)[0]
    else:
        cache = held(9, 1, past + count + 3, dim, q.dtype)
        for c, t in zip(cache, (k, v)):
            c[0, 0, :past] = t[0, :past]
            c[0, 0, past:] = NAN
        p = torch.tensor([past], dtype=torch.int32)
        out = mure.sequences([count]).attend(*cuda(q, k[:, past:], v[:, past:]), head_dim=dim, scale=scale, cache=cuda(*cache), past=p.cuda(), **how)
        expected = R.attend(q, k[:, past:], v[:, past:], [count], dim, scale=scale, cache=cache, past=p, **how)[0]
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

