"""specache_window_attend in binary16 where much of a long row's mass is in very small weights beside one large one.

A sink of small value has weight 1 and every other position 2^-a with a value of 100: what the sum loses of the small weights shows. Tolerance of a channel: the
weights' rounding h A and the final one h |o| (h = 2^-11, A = sum_j p_j |v_j|), 2^-16 A for the exponential and the binary32 sums, and for weights that binary16
holds below its smallest normal number: it takes numbers down to 2^-14 with all bits, and a weight of w times the largest is held as 2^7 w at least (2^15 w at most), so that below
w = 2^-21 it is off by 2^-25 2^-7 = 2^-32 of the largest weight at most, N 2^-32 * 100 / (sum of all) together."""
import math

import pytest
import torch

from tests.test_gpu_window import _run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("a", [10.0, 15.3, 20.1, 24.2, 25.1, 26.7, 29.9])
@pytest.mark.parametrize("n,N,window,sinks,heads", [(1, 131072, 0, 0, 2), (2, 40000, 20000, 4, 2), (1, 250, 0, 0, 2), (40, 9000, 0, 0, 2), (300, 3000, 0, 0, 2), (4096, 4096, 0, 0, 16)])
def test_many_small_weights_beside_a_large_one(n, N, window, sinks, heads, a):
    q = torch.zeros((1, heads, n, 128), device="cuda", dtype=torch.float16)
    k = torch.zeros((1, 1, N, 128), device="cuda", dtype=torch.float16)
    v = torch.full((1, 1, N, 128), 100.0, device="cuda", dtype=torch.float16)
    q[..., 3] = 4.0
    k[:, :, 0, 3] = a / 4.0                # the score in powers of two, with sm_scale = ln 2
    v[:, :, 0] = 0.1
    v[..., 64:] *= -1.0
    got = _run(q, k, v, window, sinks, sm_scale=math.log(2.0))
    scale = float(torch.tensor(math.log(2.0), dtype=torch.float32))
    x = (4.0 * k[0, 0, :, 3].double() * scale)
    p = N - n + torch.arange(n, device="cuda")[:, None]
    j = torch.arange(N, device="cuda")[None]
    seen = (j <= p) & ((j < sinks) | (p - j < window)) if window else j <= p
    w = torch.where(seen, (x - x[0]).exp()[None], 0.0)
    total = w.sum(dim=1, keepdim=True)
    want, A = (w @ v[0, 0].double()) / total, (w @ v[0, 0].double().abs()) / total
    bound = A * (2.0 ** -11 + 2.0 ** -16) + 2.0 ** -11 * want.abs() + seen.sum(dim=1, keepdim=True) * 2.0 ** -32 * 100.0 / total + 2.0 ** -25
    assert bool(((got[0].double() - want[None]).abs() <= bound[None]).all()), ((got[0].double() - want[None]).abs() - bound[None]).max().item()
