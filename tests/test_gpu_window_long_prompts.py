"""specache_window_attend on prompts long enough for workgroups of eight waves whose row tiles are so many that none is split: more than 128 row tiles of 256 rows
(a KV head's queries), each over 2048 positions or more; no scratch memory then."""
import math

import pytest
import torch

from paper_2503_16163_amd import binding
from tests.test_gpu_window import _check, _inputs, _run

pytestmark = pytest.mark.gpu
# batch, query heads, KV heads, tokens, window, sinks: 144, 304, 316 and 132 row tiles
SHAPES = [(1, 16, 16, 2300, 0, 0), (2, 16, 8, 2305, 2100, 5), (1, 32, 4, 2500, 2300, 64), (3, 11, 11, 1024, 0, 0)]


def _unsplit(B, Hq, Hkv, n, N, window, sinks):
    rows = n * (Hq // Hkv)
    walked = min(N, window + sinks + 128) if window else N
    return rows > 128 and walked >= 2048 and B * Hkv * ((rows + 255) // 256) > 128 and binding.window_scratch(B, Hq, Hkv, n, N, window, sinks) == 0


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("B,Hq,Hkv,n,window,sinks", SHAPES)
def test_whole_prompts(B, Hq, Hkv, n, window, sinks, dtype):
    N = n if n >= 2048 else 2100          # the last shape's queries stand behind what is cached
    assert _unsplit(B, Hq, Hkv, n, N, window, sinks)
    q, k, v = _inputs(n, B, Hq, Hkv, n, N, dtype)
    got = _check(q, k, v, window, sinks)
    assert torch.equal(_run(q, k, v, window, sinks, out=q), got)      # the output over the queries


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_ragged(dtype):
    """Lengths of none, one, around a row tile, and all; NaN behind every length."""
    B, Hq, Hkv, n = 6, 8, 4, 2200
    assert _unsplit(B, Hq, Hkv, n, n, 0, 0) and _unsplit(B, Hq, Hkv, n, n, 2100, 3)
    n_of, N_of = [2200, 0, 1, 129, 2049, 700], [2200, 10, 2200, 129, 2100, 300]
    q, k, v = _inputs(7, B, Hq, Hkv, n, n, dtype)
    for b in range(B):
        q[b, :, n_of[b]:] = math.nan
        k[b, :, N_of[b]:] = math.nan
        v[b, :, N_of[b]:] = math.inf
    _check(q, k, v, 0, 0, n_of, N_of)
    _check(q, k, v, 2100, 3, n_of, N_of)


@pytest.mark.parametrize("window,sinks", [(0, 0), (2050, 4)])
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_values_that_are_not_finite(dtype, window, sinks):
    Hq, Hkv, n = 16, 16, 2300
    assert _unsplit(1, Hq, Hkv, n, n, window, sinks)
    q, k, v = _inputs(8, 1, Hq, Hkv, n, n, dtype)
    clean = _run(q, k, v, window, sinks)
    v[0, 0, n - 1000, 3] = math.nan
    v[0, 1, n - 1, 100] = math.inf
    v[0, 2, 0, 7] = -math.inf
    k[0, 3, 1500] = math.nan
    got = _run(q, k, v, window, sinks)
    assert torch.equal(got[:, 4:], clean[:, 4:])
    seen = lambda at: torch.tensor([p >= at and (window == 0 or at < sinks or p - at < window) for p in range(n)], device="cuda")
    for head, at, channels in ((0, n - 1000, [3]), (1, n - 1, [100]), (2, 0, [7]), (3, 1500, list(range(128)))):
        odd = torch.zeros((n, 128), dtype=torch.bool, device="cuda")
        odd[:, channels] = seen(at)[:, None]
        assert torch.equal(got[0, head][~odd], clean[0, head][~odd]) and not bool(torch.isfinite(got[0, head][odd]).any())


def test_strides_of_a_projection():
    """Queries, keys and values as a projection leaves them, the output as the next one takes it."""
    B, Hq, Hkv, n = 1, 16, 16, 2301
    x = torch.randn((B, n, Hq + 2 * Hkv, 128), generator=torch.Generator(device="cuda").manual_seed(4), device="cuda", dtype=torch.bfloat16)
    q, k, v = (t.transpose(1, 2) for t in (x[:, :, :Hq], x[:, :, Hq:Hq + Hkv], x[:, :, Hq + Hkv:]))
    out = torch.zeros((B, n, Hq, 128), device="cuda", dtype=torch.bfloat16).transpose(1, 2)
    want = _check(q, k, v, 0, 0)
    assert torch.equal(_run(q, k, v, out=out), want)
