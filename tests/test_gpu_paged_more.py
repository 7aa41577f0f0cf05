"""Attention over pages and blocks where it can go wrong beyond its shapes: scores far from zero, values that are not finite beside positions without a page, walks of
many tiles, rows of several sequences in one tile."""
import math

import pytest
import torch

from paper_2503_16163_amd import binding
from tests.paged import attend, compare, generator, ints, pool, reference, table_of
from tests.test_gpu_blocks import _seen, attend as attend_blocks
from tests.test_gpu_window_far_scores import LEVELS

pytestmark = pytest.mark.gpu
SCALE = 1 / math.sqrt(128)


def _far(n, N, level, alike, page=32):
    """Two sequences of N positions in pages, whose scores are level times 1 to N in some order (as bfloat16 has them), or level alone; the first half shared."""
    gen = generator(n + N)
    width, shared = -(-N // page), N // 2 // page
    table, pages = table_of(gen, [N, N], page, width, shared)
    a = torch.ones(N, device="cuda") if alike else 1 + torch.randperm(N, generator=gen, device="cuda")
    scores = (level * 2.0 ** -20 * a.float()).to(torch.bfloat16)
    q = torch.zeros((2, 4, n, 128), device="cuda", dtype=torch.bfloat16)
    q[..., 5] = 2.0 ** 20
    k = torch.zeros((pages, 2, page, 128), device="cuda", dtype=torch.bfloat16)
    v = torch.randn(k.shape, generator=gen, device="cuda").to(torch.bfloat16)
    padded = torch.nn.functional.pad(scores, (0, width * page - N)).view(width, page)
    for b in range(2):
        k[table[b].long(), :, :, 5] = padded[:, None]
    return q, k, v, table, scores, shared * page


@pytest.mark.parametrize("level", LEVELS)
@pytest.mark.parametrize("n,N", [(1, 300), (2, 5000), (70, 1500), (200, 900)])
def test_far_scores(n, N, level):
    """All the weight on the largest score's positions: their value as it is, or the mean of them; behind a shared prefix and over listed blocks."""
    q, k, v, table, scores, shared = _far(n, N, level, False)
    p = N - n + torch.arange(n, device="cuda")[:, None]
    seen = torch.arange(N, device="cuda")[None] <= p
    lists = torch.arange(-(-N // 32), dtype=torch.int32, device="cuda").flip(0).expand(2, 2, n, -1).contiguous()
    cache = binding.Pages(k, v, table)
    best = torch.where(seen, scores.double()[None], -math.inf)
    best = (best == best.amax(dim=1, keepdim=True)).double()
    for got in (attend(cache, q, N, shared), attend(cache, q, N, 0), attend_blocks(cache, q, lists, N)):
        for b in range(2):
            values = v[table[b].long()].transpose(0, 1).flatten(1, 2)[:, :N].double()
            for h in range(4):
                want = (best @ values[h // 2]) / best.sum(dim=1, keepdim=True)
                # one position: its value as it is; some: their sum in binary32, divided and rounded
                bound = torch.where(best.sum(dim=1, keepdim=True) > 1, 2.0 ** -8 * want.abs() + 2.0 ** -20 * (best @ values[h // 2].abs()), torch.zeros_like(want))
                assert bool(((got[b, h].double() - want).abs() <= bound).all()), (b, h)


@pytest.mark.parametrize("level", LEVELS)
@pytest.mark.parametrize("n,N", [(2, 5000), (200, 900)])
def test_equal_far_scores(n, N, level):
    """The mean of the values seen; of +-1 and 0 all sums are exact, the result is divided and rounded."""
    q, k, v, table, _, shared = _far(n, N, level, True)
    v = v.float().sign().to(torch.bfloat16)
    seen = (torch.arange(N, device="cuda")[None] <= N - n + torch.arange(n, device="cuda")[:, None]).double()
    got = attend(binding.Pages(k, v, table), q, N, shared)
    for b in range(2):
        values = v[table[b].long()].transpose(0, 1).flatten(1, 2)[:, :N].double()
        for h in range(4):
            want = (seen @ values[h // 2]) / seen.sum(dim=1, keepdim=True)
            assert bool(((got[b, h].double() - want).abs() <= 2.0 ** -8 * want.abs() + 2.0 ** -24).all())


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("n,page", [(1, 16), (40, 64), (150, 16)])
def test_odd_values_beside_positions_without_a_page(n, page, dtype):
    """Infinities and NaN in tiles that some granules of are missing, early and late in long walks: they reach the rows that see them, and no others."""
    gen = generator(n + page)
    N_of, B, Hkv = [20000, 15001], 2, 2
    table, pages = table_of(gen, N_of, page, -(-max(N_of) // page), 1024 // page)
    k, v = pool(gen, pages, Hkv, page, dtype)
    q = torch.randn((B, 4, n, 128), generator=gen, device="cuda").to(dtype)
    first = N_of[0] - 1 - n // 2
    v[table[0, first // page].item(), 0, first % page, 7] = math.nan
    for position, channel, x in ((2000, 3, math.inf), (9000, 100, -math.inf)):       # beside the holes below
        v[table[1, position // page].item(), 1, position % page, channel] = x
    for b, position in ((0, first - page), (1, 2000 + page), (1, 9000 - page), (1, 14000), (0, 500), (1, 500)):
        table[b, position // page] = -1
    cache = binding.Pages(k, v, table)
    for shared in (0, 1024):
        exact, tol = reference(q, k, v, table, [n] * B, N_of, SCALE)
        compare(attend(cache, q, 20000, shared, None, N_of), exact, tol, [n] * B)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("Hq,n", [(64, 1), (33, 2), (40, 3)])
def test_more_rows_than_a_wave_holds(Hq, n, dtype):
    """Listed blocks for more than 32 query heads to a KV head; a list of one block, one of many."""
    gen = generator(Hq)
    N_of, page = [3000, 700], 32
    table, pages = table_of(gen, N_of, page, -(-3000 // page))
    k, v = pool(gen, pages, 1, page, dtype)
    q = torch.randn((2, Hq, n, 128), generator=gen, device="cuda").to(dtype)
    for slots in (1, 90):
        blocks = torch.stack([torch.randperm(94, generator=gen, device="cuda")[:slots] for _ in range(2 * n)]).view(2, 1, n, slots).to(torch.int32)
        exact, tol = reference(q, k, v, table, [n, n], N_of, SCALE, _seen(blocks, page, N_of))
        compare(attend_blocks(binding.Pages(k, v, table), q, blocks, 3000, None, N_of), exact, tol, [n, n])


def test_one_long_context():
    """Offsets of a table and of positions beyond what a workgroup looks up at once, a step and a part of a prompt."""
    gen = generator(2)
    N, page = 300001, 16
    table, pages = table_of(gen, [N], page, -(-N // page))
    k, v = pool(gen, pages, 1, page, torch.bfloat16)
    for n in (1, 50):
        q = torch.randn((1, 2, n, 128), generator=gen, device="cuda").to(torch.bfloat16)
        exact, tol = reference(q, k, v, table, [n], [N], SCALE)
        compare(attend(binding.Pages(k, v, table), q, N), exact, tol, [n])


def test_strides_of_tables_of_more_than_32_bits():
    gen = generator(3)
    flat = torch.full(((1 << 31) + 64,), -1, dtype=torch.int32, device="cuda")       # 8.6 GB
    table, pages = table_of(gen, [700, 650], 32, 22)
    k, v = pool(gen, pages, 2, 32, torch.float16)
    q = torch.randn((2, 4, 1, 128), generator=gen, device="cuda").half()
    far = flat.as_strided((2, 22), (1 << 31, 1))
    far.copy_(table)
    assert torch.equal(attend(binding.Pages(k, v, far), q, 700, 64, None, [700, 650]), attend(binding.Pages(k, v, table), q, 700, 64, None, [700, 650]))
