"""Rows of prompts that see positions of one half of their lanes alone (a half has places 0 to 3 of every 8, the other 4 to 7): what either half saw counts for both."""
import math

import pytest
import torch

from paper_2503_16163_amd import binding
from tests.paged import attend, compare, generator, pool, reference, table_of

pytestmark = pytest.mark.gpu
SCALE = 1 / math.sqrt(128)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("Hq,Hkv,n,N", [(2, 2, 40, 40), (8, 2, 20, 20), (8, 1, 300, 300), (16, 1, 2100, 2100)])     # tiles by 4 waves, and by 8
def test_scores_of_minus_infinity_alone(Hq, Hkv, n, N, dtype):
    """Keys of -infinity: every row has scores of -infinity alone and gives NaN in all its channels, the first four among them."""
    gen = generator(n + Hq)
    table, pages = table_of(gen, [N, N], 16, -(-N // 16))
    k, v = pool(gen, pages, Hkv, 16, dtype)
    q = torch.rand((2, Hq, n, 128), generator=gen, device="cuda").add_(0.5).to(dtype)
    k.fill_(-math.inf)
    got = attend(binding.Pages(k, v, table), q, N)
    assert bool(torch.isnan(got[:, :, :8]).all()) and bool(torch.isnan(got).all())


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("Hq,Hkv,n", [(2, 2, 40), (8, 2, 20)])
def test_some_heads_scores_of_minus_infinity(Hq, Hkv, n, dtype):
    """One KV head's keys of -infinity, the first page missing: rows on it see nothing and give zeros, the next four see one half's places alone."""
    gen = generator(n)
    N = n + 16
    table, pages = table_of(gen, [N], 16, -(-N // 16))
    k, v = pool(gen, pages, Hkv, 16, dtype)
    q = torch.rand((1, Hq, N, 128), generator=gen, device="cuda").add_(0.5).to(dtype)
    table[0, 0] = -1
    k[:, 1] = -math.inf
    got = attend(binding.Pages(k, v, table), q, N)
    G = Hq // Hkv
    assert bool((got[:, :, :16] == 0).all()) and bool(torch.isnan(got[:, G:, 16:]).all())
    exact, tol = reference(q[:, :G], k[:, :1], v[:, :1], table, [N], [N], SCALE)
    compare(got[:, :G], exact, tol, [N])
