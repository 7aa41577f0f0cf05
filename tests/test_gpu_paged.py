"""specache_paged_attend against the definition in 64 bits, row by row."""
import math

import pytest
import torch

from paper_2503_16163_amd import binding
from tests.paged import attend, compare, generator, ints, pool, reference, scratch_of, table_of

pytestmark = pytest.mark.gpu
SCALE = 1 / math.sqrt(128)


def _make(seed, B, Hq, Hkv, n, N_of, page, shared, dtype, order="heads", width=None):
    gen = generator(seed)
    width = -(-max(N_of) // page) if width is None else width
    table, pages = table_of(gen, N_of, page, max(width, 1), shared // page)
    k, v = pool(gen, pages, Hkv, page, dtype, order)
    q = torch.randn((B, Hq, n, 128), generator=gen, device="cuda").to(dtype)
    return q, k, v, table


def _check(q, k, v, table, kv_tokens, shared, n_of, N_of, sm_scale=0.0):
    B = q.shape[0]
    cache = binding.Pages(k, v, table)
    got = attend(cache, q, kv_tokens, shared, n_of, N_of, sm_scale)
    n, N = n_of or [q.shape[2]] * B, N_of or [kv_tokens] * B
    exact, tol = reference(q, k, v, table, n, N, sm_scale or SCALE)
    compare(got, exact, tol, n)
    return got


SHAPES = [  # B, Hq, Hkv, n, N_of, page, shared
    (1, 1, 1, 1, [1], 16, 0), (2, 2, 1, 1, [63, 1], 16, 0), (1, 4, 4, 1, [64], 32, 0), (3, 8, 2, 1, [65, 33, 64], 64, 0), (1, 32, 8, 2, [5003], 16, 0),
    (2, 64, 1, 1, [2500, 777], 128, 0), (2, 16, 2, 4, [9000, 4], 256, 0), (1, 2, 2, 31, [31], 16, 0), (2, 6, 2, 129, [129, 129], 64, 0), (1, 8, 2, 256, [4096], 32, 0),
    (3, 6, 3, 150, [2500, 150, 700], 16, 0), (1, 8, 8, 520, [520], 64, 0), (2, 2, 2, 40, [7, 90], 16, 0),
    (2, 2, 1, 1, [64, 50], 16, 32), (3, 32, 32, 1, [1200, 1001, 1100], 16, 1000), (16, 8, 2, 1, [700 + 13 * i for i in range(16)], 64, 650),
    (5, 64, 8, 2, [3000, 2050, 2049, 2100, 2500], 32, 2049), (64, 4, 1, 1, [5000 + 7 * i for i in range(64)], 64, 4999), (33, 8, 8, 3, [400 + i for i in range(33)], 16, 390),
    (4, 8, 2, 70, [1070, 1100, 1500, 1071], 16, 1000), (3, 16, 2, 200, [2500, 2300, 2248], 64, 2100), (2, 8, 4, 300, [350, 400], 32, 100), (2, 4, 4, 20, [5000, 4981], 256, 4900),
    (8, 8, 1, 40, [4200 + 11 * i for i in range(8)], 128, 4100),
]


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("B,Hq,Hkv,n,N_of,page,shared", SHAPES)
def test_paged_attend(B, Hq, Hkv, n, N_of, page, shared, dtype):
    q, k, v, table = _make(n * 7 + N_of[0], B, Hq, Hkv, n, N_of, page, shared, dtype, "places" if n % 2 else "heads")
    got = _check(q, k, v, table, max(N_of), shared, None, N_of)
    if shared:                      # sharing changes the rounding alone
        alone = attend(binding.Pages(k, v, table), q, max(N_of), 0, None, N_of)
        exact, tol = reference(q, k, v, table, [n] * B, N_of, SCALE)
        compare(alone, exact, tol, [n] * B)
        assert got.shape == alone.shape


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("n,page,n_of,N_of,shared", [
    (1, 16, [1, 0, 1, 1], [700, 5, 0, 1], 0), (2, 64, [2, 1, 2, 0], [9000, 64, 1, 77], 0), (260, 32, [260, 1, 0, 131], [260, 1, 0, 131], 0),
    (3, 16, [3, 3, 3, 3], [0, 1, 2, 5000], 0), (150, 64, [150, 20, 150, 3], [400, 10, 150, 399], 0),
    # sequences that end inside what is shared, or have no queries, or nothing at all
    (1, 16, [1, 0, 1, 1], [700, 500, 0, 100], 640), (2, 32, [2, 1, 2, 0], [3000, 64, 1, 2999], 2900), (90, 64, [90, 1, 0, 31], [1000, 970, 960, 200], 960),
    (200, 16, [200, 200, 3, 150], [900, 60, 2, 512], 500)])
def test_ragged_batches(n, page, n_of, N_of, shared, dtype):
    """Lengths of zero, fewer cached tokens than queries; what is behind the lengths holds NaN, in pages that are named all the same."""
    B, width = 4, -(-max(N_of) // page) + 1
    q, k, v, table = _make(n + N_of[0], B, 8, 2, n, [width * page] * B, page, shared, dtype)
    for b in range(B):
        q[b, :, n_of[b]:] = math.nan
        for i in range(max(N_of[b], shared // page * page) // page, width):
            keep = max(0, N_of[b] - i * page)
            k[table[b, i].item(), :, keep:] = math.nan
            v[table[b, i].item(), :, keep:] = math.inf
    _check(q, k, v, table, width * page, shared, n_of, N_of)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("n,shared", [(1, 0), (3, 512), (100, 0), (100, 512)])
def test_entries_that_name_no_page(n, shared, dtype):
    """Positions without a page are seen by nobody, whatever lies about; a sequence with no page at all gives zeros."""
    N_of, page = [1500, 1333, 900], 32
    q, k, v, table = _make(5 + n, 3, 8, 2, n, N_of, page, shared, dtype)
    table[:, 3] = -1                                   # of what is shared, alike
    table[:, 7] = 2 ** 31 - 1
    table[0, 20] = k.shape[0]
    table[1, 39:] = -(2 ** 31)
    table[2, 24:] = -5
    if not shared:
        table[2] = -1
    _check(q, k, v, table, 1500, shared, None, N_of)
    cache = binding.Pages(k[:0], v[:0], table)
    assert bool((attend(cache, q, 1500, shared, None, N_of) == 0).all())


def test_lengths_are_held_to_the_counts():
    q, k, v, table = _make(5, 3, 2, 2, 4, [112] * 3, 16, 0, torch.float16)
    cache = binding.Pages(k, v, table)
    assert torch.equal(attend(cache, q, 100, 0, [9, -3, 4], [1000, 50, -1]), attend(cache, q, 100, 0, [4, 0, 4], [100, 50, 0]))


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("n,N,shared", [(200, 200, 0), (3, 2000, 1024), (70, 1500, 1024), (2, 700, 0)])
def test_values_that_are_not_finite_reach_the_rows_that_see_them_alone(n, N, shared, dtype):
    q, k, v, table = _make(n, 2, 4, 2, n, [N, N], 64, shared, dtype)
    def at(b, j):
        return table[b, j // 64].item(), j % 64
    p, s = at(0, N - n // 2 - 1)
    v[p, 0, s, 3] = math.nan
    p, s = at(0, N - 1)
    v[p, 1, s, 100] = math.inf
    p, s = at(1, N - 1)
    v[p, 1, s, 7] = -math.inf
    _check(q, k, v, table, N, shared, None, [N, N])
    clean = v.nan_to_num(0, 0, 0)
    k2 = k.clone()
    p, s = at(0, N - 1)
    k2[p, 1, s] = math.nan
    a, b = (attend(binding.Pages(x, clean, table), q, N, shared) for x in (k, k2))
    assert torch.equal(a[1], b[1]) and torch.equal(a[0, :2], b[0, :2]) and torch.equal(a[0, :, :n - 1], b[0, :, :n - 1]) and bool(torch.isnan(b[0, 2:, n - 1]).all())


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_scores_over_the_whole_range(dtype):
    q, k, v, table = _make(11, 2, 4, 2, 90, [900, 800], 16, 320, dtype)
    _check(q * 20, k, v, table, 900, 320, None, [900, 800])
    _check(q * 20, k, v, table, 900, 320, None, [900, 800], sm_scale=0.003)
    q, k, v, table = _make(12, 2, 2, 1, 2, [4000, 3900], 64, 2048, dtype)
    rising = torch.linspace(0, 4, 4032, device="cuda").view(-1, 64)
    for b in range(2):
        for i in range(63):
            if table[b, i] >= 0:
                k[table[b, i].item()] = (q[0, :1, :1] * rising[i][None, :, None]).to(dtype)
    _check(q, k, v, table, 4000, 2048, None, [4000, 3900])
    _check(q, torch.zeros_like(k), v, table, 4000, 2048, None, [4000, 3900])
    # the whole prefix at scores of -infinity, then everything
    minus = k.clone()
    minus[table[0, :32].long()] = -math.inf
    q = q.abs() + 0.5
    got = _check(q, minus, v, table, 4000, 2048, None, [4000, 3900])
    assert bool(torch.isfinite(got).all())
    minus.fill_(-math.inf)
    assert bool(torch.isnan(attend(binding.Pages(minus, v, table), q, 4000, 2048, None, [4000, 3900])).all())


def test_views_of_all_kinds():
    """Fused keys and values, the output over q, tables whose rows lie apart, a table row for all."""
    gen = generator(3)
    pages = torch.randn((40, 2, 32, 2, 128), generator=gen, device="cuda").to(torch.bfloat16)       # [page, KV head, place, k or v]
    k, v = pages[:, :, :, 0], pages[:, :, :, 1]
    wide = torch.full((3, 50), -1, dtype=torch.int32, device="cuda")
    wide[:, :12] = torch.randperm(40, generator=gen, device="cuda")[:36].view(3, 12).to(torch.int32)
    table = wide[:, :12]
    q = torch.randn((3, 7, 8, 128), generator=gen, device="cuda").to(torch.bfloat16).transpose(1, 2)
    cache = binding.Pages(k, v, table)
    want = attend(cache, q.contiguous(), 380, 0)
    exact, tol = reference(q, k, v, table, [7] * 3, [380] * 3, SCALE)
    compare(want, exact, tol, [7] * 3)
    assert torch.equal(attend(cache, q, 380, 0), want)
    mine = q.clone()
    assert torch.equal(attend(cache, mine, 380, 0, out=mine), want)
    same = table[:1].expand(3, -1)
    assert torch.equal(attend(binding.Pages(k, v, same), q, 380, 0), attend(binding.Pages(k, v, same.contiguous()), q, 380, 0))


def test_pages_beyond_32_bit_offsets():
    flat = torch.empty((5 << 30) // 2 * 2, device="cuda", dtype=torch.float16)      # 10 GB
    n_pages, page = 40, 64
    far = flat.as_strided((n_pages, 2, page, 128), (1 << 27, page * 128, 128, 1))
    q, k, v, table = _make(8, 2, 4, 2, 2, [1200, 1100], page, 512, torch.float16)
    table = table % n_pages
    k, v = k[:n_pages].contiguous(), v[:n_pages].contiguous()
    assert k.shape[0] == n_pages or k.shape[0] < n_pages
    far = far[:k.shape[0]]
    far.copy_(k)
    assert torch.equal(attend(binding.Pages(far, v, table), q, 1200, 512), attend(binding.Pages(k, v, table), q, 1200, 512))
    q = torch.randn((2, 4, 90, 128), device="cuda").half()
    assert torch.equal(attend(binding.Pages(far, v, table), q, 1200, 512), attend(binding.Pages(k, v, table), q, 1200, 512))


@pytest.mark.parametrize("B,Hq,Hkv,n,N,shared", [(2, 8, 2, 2, 9000, 4096), (4, 4, 4, 100, 1300, 1000), (3, 8, 8, 1, 300, 0)])
def test_captured_overlapping_and_the_same_every_time(B, Hq, Hkv, n, N, shared):
    """Two graphs with scratch memory of their own, replayed on two streams at a time between eager calls; lengths and tables move between replays."""
    sets = []
    for i in range(2):
        q, k, v, table = _make(20 + i, B, Hq, Hkv, n, [N] * B, 32, shared, torch.bfloat16)
        cache = binding.Pages(k, v, table)
        s = dict(q=q, cache=cache, table=table, out=torch.zeros_like(q), scratch=scratch_of(binding.paged_scratch(cache, B, Hq, n, N, shared)),
                 N=torch.full((B,), N, dtype=torch.int32, device="cuda"), stream=torch.cuda.Stream(), graph=torch.cuda.CUDAGraph())
        torch.cuda.synchronize()
        with torch.cuda.graph(s["graph"], stream=s["stream"]):
            binding.paged_attend(cache, q, s["out"], N, shared, kv_lengths=s["N"], scratch=s["scratch"])
        sets.append(s)
    for turn in range(3):
        for s in sets:
            s["q"].copy_(torch.randn_like(s["q"]))
            s["N"].fill_(N - 13 * turn)
            s["table"][:, shared // 32:] = s["table"][:, shared // 32:].roll(1, dims=0)
        want = [attend(s["cache"], s["q"], N, shared, N_of=s["N"].tolist()) for s in sets]
        torch.cuda.synchronize()
        for s in sets:
            with torch.cuda.stream(s["stream"]):
                s["graph"].replay()
        torch.cuda.synchronize()
        for s, w in zip(sets, want):
            assert torch.equal(s["out"], w)
