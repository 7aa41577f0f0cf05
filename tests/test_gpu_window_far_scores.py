"""specache_window_attend where the scores that a row sees are far from zero, on either side: the softmax is that of their differences all the same.

One channel makes the scores, whole multiples of a large power of two: the differences leave all the weight on the largest, so the output is that
position's value, bit for bit; equal scores give the mean of the values (of +-1 and 0, so that every sum is exact)."""
import math

import pytest
import torch

from tests.test_gpu_window import _run

pytestmark = pytest.mark.gpu
SHAPES = [(1, 300, 0, 0), (2, 5000, 0, 0), (2, 5000, 700, 4), (70, 70, 0, 0), (200, 1500, 90, 3), (300, 2600, 0, 0)]


LEVELS = [-2.0 ** 115, -2.0 ** 101, -2.0 ** 60, -2.0 ** 40, -2.0 ** 28, 2.0 ** 28, 2.0 ** 40, 2.0 ** 60, 2.0 ** 115]


def _inputs(n, N, level, alike):
    """Scores of level times 1 to N (as bfloat16 has them), or of level alone, before sm_scale."""
    q = torch.zeros((2, 4, n, 128), device="cuda", dtype=torch.bfloat16)
    k = torch.zeros((2, 2, N, 128), device="cuda", dtype=torch.bfloat16)
    q[..., 5] = 2.0 ** 20
    gen = torch.Generator(device="cuda")
    gen.manual_seed(n + N)
    a = torch.ones(N, device="cuda") if alike else 1 + torch.randperm(N, generator=gen, device="cuda")
    k[..., 5] = (level * 2.0 ** -20 * a.float()).to(torch.bfloat16)
    v = torch.randn((2, 2, N, 128), generator=gen, device="cuda").to(torch.bfloat16)
    return q, k, v


def _seen(n, N, window, sinks):
    p = N - n + torch.arange(n, device="cuda")[:, None]
    j = torch.arange(N, device="cuda")[None]
    s = j <= p
    return s & ((j < sinks) | (p - j < window)) if window else s


@pytest.mark.parametrize("level", LEVELS)
@pytest.mark.parametrize("n,N,window,sinks", SHAPES)
def test_the_largest_of_far_scores(n, N, window, sinks, level):
    q, k, v = _inputs(n, N, level, False)
    got = _run(q, k, v, window, sinks)
    x = torch.where(_seen(n, N, window, sinks), k[0, 0, :, 5].double()[None], -math.inf)
    best = (x == x.amax(dim=1, keepdim=True)).double()
    for b in range(2):
        for h in range(4):
            values = v[b, h // 2].double()
            want = (best @ values) / best.sum(dim=1, keepdim=True)
            # one position: its value as it is; some: their sum in binary32, divided and rounded
            bound = torch.where(best.sum(dim=1, keepdim=True) > 1, 2.0 ** -8 * want.abs() + 2.0 ** -20 * (best @ values.abs()), torch.zeros_like(want))
            assert bool(((got[b, h].double() - want).abs() <= bound).all()), (b, h)


@pytest.mark.parametrize("level", LEVELS)
@pytest.mark.parametrize("n,N,window,sinks", SHAPES)
def test_equal_far_scores(n, N, window, sinks, level):
    q, k, v = _inputs(n, N, level, True)
    v = v.float().sign().to(torch.bfloat16)
    got = _run(q, k, v, window, sinks)
    seen = _seen(n, N, window, sinks).double()
    for b in range(2):
        for h in range(4):
            want = (seen @ v[b, h // 2].double()) / seen.sum(dim=1, keepdim=True)
            assert bool(((got[b, h].double() - want).abs() <= 2.0 ** -8 * want.abs() + 2.0 ** -22).all())


@pytest.mark.parametrize("n,N,window,sinks", SHAPES)
def test_only_scores_of_minus_infinity(n, N, window, sinks):
    """No softmax has these, so the rows that see nothing else are NaN, as in the definition; a row that sees one finite score has that position's value."""
    q, k, v = _inputs(n, N, -1.0, True)
    q[..., 5] = 1.0
    k[..., 5] = -math.inf
    assert bool(torch.isnan(_run(q, k, v, window, sinks)).all())
    k[:, :, N - 1, 5] = -3.0
    got = _run(q, k, v, window, sinks)
    assert bool(torch.isnan(got[:, :, :n - 1]).all())
    assert torch.equal(got[:, :, n - 1], v[:, :, N - 1].repeat_interleave(2, dim=1))
    # rows that see nothing stay zeros
    got = _run(q, k[:, :, :1].contiguous(), v[:, :, :1].contiguous())
    assert bool((got[:, :, :n - 1] == 0).all()) and bool(torch.isnan(got[:, :, n - 1]).all())


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("n,N,window,sinks", SHAPES)
def test_an_infinite_key_reaches_the_rows_that_see_it_alone(n, N, window, sinks, dtype):
    """Rows beside such a row, in one wave with it, keep every bit."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(n)
    q, k, v = (torch.randn(s, generator=gen, device="cuda").to(dtype) for s in ((1, 4, n, 128), (1, 2, N, 128), (1, 2, N, 128)))
    odd = k.clone()
    odd[0, 1, N - 1, 9] = math.inf
    q[..., 9] = q[..., 9].abs() + 0.5
    clean, got = _run(q, k, v, window, sinks), _run(q, odd, v, window, sinks)
    assert torch.equal(clean[:, :2], got[:, :2]) and torch.equal(clean[:, :, :n - 1], got[:, :, :n - 1])
    assert bool(torch.isnan(got[:, 2:, n - 1]).all())
