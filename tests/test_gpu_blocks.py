"""specache_block_select and specache_block_attend: lists equal to the definition's in 64 bits, attention within its tolerance."""
import math

import pytest
import torch

from paper_2503_16163_amd import binding
from tests.paged import compare, generator, ints, pool, reference, scratch_of, table_of

pytestmark = pytest.mark.gpu
SCALE = 1 / math.sqrt(128)


def bounds_of(k):
    return torch.stack([k.amin(dim=2), k.amax(dim=2)], dim=2).contiguous()


def lists(q, bounds, table, n_of, N_of, page, top, first, recent):
    """The definition, a row at a time, in 64 bits."""
    B, Hq, n_all, _ = q.shape
    P, Hkv = bounds.shape[:2]
    G = Hq // Hkv
    out = torch.full((B, Hkv, n_all, top + first + recent), -1, dtype=torch.int32)
    for b in range(B):
        n, N = n_of[b], N_of[b]
        for h in range(Hkv):
            for i in range(n):
                p = N - n + i
                if p < 0:
                    continue
                row = table[b, :p // page + 1].long()
                there = ((row >= 0) & (row < P)).cpu()
                low, high = (bounds[row.clamp(0, max(P - 1, 0)), h, x].double() for x in (0, 1))
                score = torch.full((len(row),), -math.inf, dtype=torch.float64, device=q.device)
                for g in range(h * G, h * G + G):
                    x = q[b, g, i].double()
                    one = (x.clamp(min=0) * high + x.clamp(max=0) * low).sum(dim=1)
                    score = torch.maximum(score, torch.where(torch.isnan(one), -math.inf, one))
                score = score.cpu()
                always = [c for c in range(len(row)) if there[c] and (c < first or c > p // page - recent)]
                rest = sorted((c for c in range(len(row)) if there[c] and c not in set(always)), key=lambda c: (-score[c].item(), c))[:top]
                ids = sorted(always + rest)
                out[b, h, i, :len(ids)] = torch.tensor(ids, dtype=torch.int32)
    return out.cuda()


def select(cache, q, kv_tokens, top, first, recent, n_of=None, N_of=None, stream=None):
    B, Hq, n, _ = q.shape
    blocks = torch.full((B, cache.config.n_kv_heads, n, top + first + recent), -9, dtype=torch.int32, device="cuda")
    scratch = scratch_of(binding.block_scratch(cache, B, Hq, n, kv_tokens, top, first, recent))
    binding.block_select(cache, q, blocks, kv_tokens, top, first, recent, ints(n_of), ints(N_of), scratch, stream)
    return blocks


def attend(cache, q, blocks, kv_tokens, n_of=None, N_of=None, sm_scale=0.0, out=None):
    B, Hq, n, _ = q.shape
    out = torch.full(q.shape, 7.0, device="cuda", dtype=q.dtype) if out is None else out
    scratch = scratch_of(binding.block_scratch(cache, B, Hq, n, kv_tokens, blocks.shape[3]))
    binding.block_attend(cache, q, out, blocks, kv_tokens, ints(n_of), ints(N_of), sm_scale, scratch)
    return out


def _seen(blocks, page, N_of):
    def of(b, h):
        N = N_of[b]
        seen = torch.zeros((blocks.shape[2], -(-N // page) + 1), dtype=torch.bool, device="cuda")
        l = blocks[b, h].long()
        seen.scatter_(1, torch.where((l >= 0) & (l < seen.shape[1]), l, seen.shape[1] - 1), True)
        seen[:, -1] = False
        return seen[:, :-1].repeat_interleave(page, dim=1)[:, :N]
    return of


def _make(seed, B, Hq, Hkv, n, N_of, page, dtype, order="heads"):
    gen = generator(seed)
    table, pages = table_of(gen, N_of, page, max(-(-max(N_of) // page), 1))
    k, v = pool(gen, pages, Hkv, page, dtype, order)
    k = k + torch.randn((pages, Hkv, 1, 128), generator=gen, device="cuda").to(dtype) * 0.5
    q = torch.randn((B, Hq, n, 128), generator=gen, device="cuda").to(dtype)
    return q, k, v, bounds_of(k), table


SHAPES = [  # B, Hq, Hkv, n, N_of, page, top, first, recent
    (1, 1, 1, 1, [1], 16, 1, 0, 0), (2, 4, 1, 1, [300, 17], 16, 4, 1, 2), (1, 32, 32, 2, [2000], 16, 20, 1, 4), (3, 8, 2, 1, [5000, 4999, 64], 64, 8, 0, 1),
    (1, 64, 1, 3, [1000], 32, 5, 2, 0), (2, 20, 1, 2, [700, 555], 128, 2, 1, 1), (1, 3, 3, 20, [900], 16, 7, 1, 2), (2, 8, 2, 33, [600, 40], 32, 3, 0, 0),
    (1, 8, 4, 1, [20000], 16, 64, 4, 8), (1, 2, 1, 1, [70000], 16, 100, 1, 1), (1, 4, 2, 2, [3000], 256, 1, 0, 0), (2, 4, 2, 1, [800, 90], 16, 0, 2, 3), (1, 2, 2, 1, [500], 16, 200, 3, 3),
    (1, 16, 1, 17, [333], 64, 2, 0, 1), (1, 48, 2, 2, [900], 16, 9, 1, 1), (1, 2, 1, 1, [150000], 16, 30, 1, 1),
]


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("B,Hq,Hkv,n,N_of,page,top,first,recent", SHAPES)
def test_blocks(B, Hq, Hkv, n, N_of, page, top, first, recent, dtype):
    q, k, v, bounds, table = _make(N_of[0] + n, B, Hq, Hkv, n, N_of, page, dtype, "places" if n % 2 else "heads")
    cache = binding.Pages(k, v, table, bounds)
    got = select(cache, q, max(N_of), top, first, recent, None, N_of)
    assert torch.equal(got, lists(q, bounds, table, [n] * B, N_of, page, top, first, recent))
    exact, tol = reference(q, k, v, table, [n] * B, N_of, SCALE, _seen(got, page, N_of))
    compare(attend(cache, q, got, max(N_of), None, N_of), exact, tol, [n] * B)


def test_scores_bound_what_the_blocks_hold():
    """A block that is not chosen holds no score above the bound of the worst one chosen."""
    q, k, v, bounds, table = _make(4, 1, 4, 1, 1, [1600], 16, torch.bfloat16)
    got = select(binding.Pages(k, v, table, bounds), q, 1600, 10, 0, 0)[0, 0, 0].tolist()
    b = bounds[table[0].long(), 0].double()
    bound = torch.stack([(q[0, g, 0].double().clamp(min=0) * b[:, 1] + q[0, g, 0].double().clamp(max=0) * b[:, 0]).sum(1) for g in range(4)]).amax(0)
    real = torch.einsum("gc,pjc->pgj", q[0, :, 0].double().cpu(), k[table[0].long(), 0].double().cpu()).amax(dim=(1, 2)).cuda()
    assert bool((real <= bound).all())
    worst = bound[got].min()
    assert all(real[c] <= worst for c in range(100) if c not in got)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_equal_scores_take_the_lower_block(dtype):
    q, k, v, bounds, table = _make(6, 2, 4, 2, 2, [1600, 1599], 16, dtype)
    for level in (0, 3, 40):       # all alike, a few above the others, all of either sign
        some = bounds.clone()
        some[:] = bounds[:1]
        some[table[:, :level].long()] = bounds[1]
        cache = binding.Pages(k, v, table, some)
        got = select(cache, q, 1600, 11, 1, 2, None, [1600, 1599])
        assert torch.equal(got, lists(q, some, table, [2, 2], [1600, 1599], 16, 11, 1, 2))
    zero = torch.zeros_like(bounds)
    zero[::2] *= -1.0
    cache = binding.Pages(k, v, table, zero)
    assert torch.equal(select(cache, q, 1600, 5, 0, 1, None, [1600, 1599]), lists(q, zero, table, [2, 2], [1600, 1599], 16, 5, 0, 1))


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_neighbouring_scores(dtype):
    """Blocks that differ in the last bit of one channel, and sums whose addends differ by 2^20: what binary32 sums would confuse."""
    q, k, v, bounds, table = _make(7, 1, 2, 1, 1, [3200], 16, dtype)
    some = bounds[:1].repeat(bounds.shape[0], 1, 1, 1)
    some[:, :, :, 5] = 512.0
    some[:, :, :, 6] = -512.0
    q[:, :, :, 5] = q[:, :, :, 6] = 100.0
    q[:, :, :, 9] = 2.0 ** -10
    steps = torch.randint(0, 100, (bounds.shape[0], 1), generator=generator(1), device="cuda")
    some[:, :, 0, 9] = some[:, :, 1, 9] = (1 + steps * 2.0 ** -7).to(dtype)
    got = select(binding.Pages(k, v, table, some), q, 3200, 40, 0, 0)
    assert torch.equal(got, lists(q, some, table, [1], [3200], 16, 40, 0, 0))


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("N,top", [(4000, 30), (9600, 300), (30000, 100), (100000, 600), (300000, 50)])
def test_many_scores_alike(N, top, dtype):
    """More blocks near to the last chosen one than are told apart in LDS: all of them equal, in a few steps, or different in their last bits alone."""
    q, k, v, bounds, table = _make(8, 1, 2, 1, 1, [N], 16, dtype)
    gen, P = generator(2), bounds.shape[0]
    one = bounds[:1].repeat(P, 1, 1, 1)
    steps = one.clone()
    steps[:, :, :, 4] = torch.randint(-2, 3, (P, 1, 1), generator=gen, device="cuda").to(dtype)
    close = one.clone()
    close[:, :, :, 5], close[:, :, :, 6] = 512.0, -512.0
    close[:, :, :, 9] = (1 + torch.randint(0, 100, (P, 1, 1), generator=gen, device="cuda") * 2.0 ** -7).to(dtype)
    x = q.clone()
    x[:, :, :, 5] = x[:, :, :, 6] = 100.0
    x[:, :, :, 9] = 2.0 ** -10
    mixed = torch.where((torch.arange(P, device="cuda") % 3 == 0)[:, None, None, None], bounds, one)
    for queries, some in ((q, one), (q, steps), (x, close), (q, mixed), (q, torch.zeros_like(one))):
        cache = binding.Pages(k, v, table, some)
        assert torch.equal(select(cache, queries, N, top, 1, 2), lists(queries, some, table, [1], [N], 16, top, 1, 2))


def test_smallest_and_largest_numbers():
    """Bounds and queries below the smallest normal number, and products beyond the largest of 32 bits."""
    for dtype, scales in ((torch.float16, (2.0 ** -22, 2.0 ** 14)), (torch.bfloat16, (1e-38, 1e38))):
        for scale in scales:
            q, k, v, bounds, table = _make(13, 1, 4, 2, 2, [3200], 16, dtype)
            some, x = (bounds.double() * scale).to(dtype), (q.double() * scale).to(dtype)
            for top in (7, 100):
                assert torch.equal(select(binding.Pages(k, v, table, some), x, 3200, top, 1, 1), lists(x, some, table, [2], [3200], 16, top, 1, 1))


@pytest.mark.parametrize("n,n_of,N_of", [(1, [1, 0, 1, 1], [700, 5, 0, 1]), (3, [3, 3, 2, 0], [2, 1, 900, 77]), (40, [40, 1, 39, 20], [30, 900, 39, 500])])
def test_ragged_batches_and_missing_pages(n, n_of, N_of):
    q, k, v, bounds, table = _make(n, 4, 8, 2, n, [912] * 4, 16, torch.bfloat16)
    table[:, 4] = -1
    table[1, 20:23] = 2 ** 31 - 1
    table[2, 0] = k.shape[0]
    for b in range(4):             # behind a sequence's tokens, anything
        q[b, :, n_of[b]:] = math.nan
        for i in range(-(-N_of[b] // 16), 57):
            if i != 4 and 0 <= table[b, i] < k.shape[0]:
                k[table[b, i].item()] = math.nan
                bounds[table[b, i].item()] = math.nan
    cache = binding.Pages(k, v, table, bounds)
    for top, first, recent in ((6, 1, 2), (3, 6, 0), (60, 0, 0)):
        got = select(cache, q, 912, top, first, recent, n_of, N_of)
        want = lists(q, bounds, table, n_of, N_of, 16, top, first, recent)
        for b in range(4):
            assert torch.equal(got[b, :, :n_of[b]], want[b, :, :n_of[b]]) and bool((got[b, :, n_of[b]:] == -9).all())
        exact, tol = reference(q, k, v, table, n_of, N_of, SCALE, lambda b, h: _seen(want, 16, N_of)(b, h)[:n_of[b]])
        compare(attend(cache, q, got.clamp(min=-1), 912, n_of, N_of), exact, tol, n_of)


def test_bounds_that_are_not_finite():
    q, k, v, bounds, table = _make(9, 1, 4, 2, 2, [800], 16, torch.float16)
    bounds[table[0, 3].item(), :, 1, 7] = math.nan
    bounds[table[0, 5].item(), 0] = math.inf
    bounds[table[0, 8].item(), :, 0] = -math.inf
    bounds[table[0, 9].item(), :, 1] = -math.inf
    q[0, 1, 1, 3] = math.nan
    for top in (5, 46, 60):
        assert torch.equal(select(binding.Pages(k, v, table, bounds), q, 800, top, 1, 1), lists(q, bounds, table, [2], [800], 16, top, 1, 1))


def test_lists_of_the_callers_own():
    """In any order, with entries that are no block, a block that is later than the row, and one that counts twice."""
    q, k, v, bounds, table = _make(10, 2, 4, 2, 2, [500, 77], 16, torch.bfloat16)
    cache = binding.Pages(k, v, table)
    blocks = torch.full((2, 2, 2, 9), -1, dtype=torch.int32, device="cuda")
    blocks[..., 0], blocks[..., 2], blocks[..., 3], blocks[..., 5], blocks[..., 6] = 4, 2, 0, 2 ** 31 - 1, 31
    blocks[..., 7] = -(2 ** 31)
    exact, tol = reference(q, k, v, table, [2, 2], [500, 77], SCALE, _seen(blocks, 16, [500, 77]))
    compare(attend(cache, q, blocks, 500, None, [500, 77]), exact, tol, [2, 2])
    # twice: as if the block's positions stood there twice
    twice = torch.tensor([1, 3, 1], dtype=torch.int32, device="cuda").expand(2, 2, 2, 3).contiguous()
    again = table.clone()
    again[:, 0] = table[:, 1]      # the same page as a block of its own
    other = torch.tensor([0, 1, 3], dtype=torch.int32, device="cuda").expand(2, 2, 2, 3).contiguous()
    got, want = attend(cache, q, twice, 500, None, [500, 77]), attend(binding.Pages(k, v, again), q, other, 500, None, [500, 77])
    exact, tol = reference(q, k, v, again, [2, 2], [500, 77], SCALE, _seen(other, 16, [500, 77]))
    compare(got, exact, tol, [2, 2])
    compare(want, exact, tol, [2, 2])
    assert bool((attend(cache, q, torch.full_like(twice, -1), 500, None, [500, 77]) == 0).all())


def test_all_blocks_are_paged_attention():
    from tests.paged import attend as whole
    q, k, v, bounds, table = _make(12, 2, 8, 2, 5, [1000, 300], 32, torch.float16)
    cache = binding.Pages(k, v, table, bounds)
    got = select(cache, q, 1000, 32, 0, 0, None, [1000, 300])
    a, b = attend(cache, q, got, 1000, None, [1000, 300]), whole(cache, q, 1000, 0, None, [1000, 300])
    exact, tol = reference(q, k, v, table, [5, 5], [1000, 300], SCALE)
    compare(a, exact, tol, [5, 5])
    compare(b, exact, tol, [5, 5])


@pytest.mark.parametrize("B,Hq,Hkv,n,N,page,top", [(2, 8, 2, 2, 9000, 16, 40), (1, 4, 4, 30, 700, 32, 5)])
def test_captured_overlapping_and_the_same_every_time(B, Hq, Hkv, n, N, page, top):
    sets = []
    for i in range(2):
        q, k, v, bounds, table = _make(20 + i, B, Hq, Hkv, n, [N] * B, page, torch.bfloat16)
        cache = binding.Pages(k, v, table, bounds)
        s = dict(q=q, cache=cache, out=torch.zeros_like(q), scratch=scratch_of(binding.block_scratch(cache, B, Hq, n, N, top, 1, 2)),
                 blocks=torch.zeros((B, Hkv, n, top + 3), dtype=torch.int32, device="cuda"), N=torch.full((B,), N, dtype=torch.int32, device="cuda"),
                 stream=torch.cuda.Stream(), graph=torch.cuda.CUDAGraph())
        torch.cuda.synchronize()
        with torch.cuda.graph(s["graph"], stream=s["stream"]):
            binding.block_select(cache, q, s["blocks"], N, top, 1, 2, kv_lengths=s["N"], scratch=s["scratch"])
            binding.block_attend(cache, q, s["out"], s["blocks"], N, kv_lengths=s["N"], scratch=s["scratch"])
        sets.append(s)
    for turn in range(3):
        for s in sets:
            s["q"].copy_(torch.randn_like(s["q"]))
            s["N"].fill_(N - 13 * turn)
        want = []
        for s in sets:
            blocks = select(s["cache"], s["q"], N, top, 1, 2, N_of=s["N"].tolist())
            want.append((blocks, attend(s["cache"], s["q"], blocks, N, N_of=s["N"].tolist())))
        torch.cuda.synchronize()
        for s in sets:
            with torch.cuda.stream(s["stream"]):
                s["graph"].replay()
        torch.cuda.synchronize()
        for s, (blocks, out) in zip(sets, want):
            assert torch.equal(s["blocks"], blocks) and torch.equal(s["out"], out)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("B,Hq,Hkv,n,N_of,page,top,first,recent", [
    # units for one, two and four waves to a workgroup; few chunks, which one wave joins
    (2, 16, 8, 150, [700, 333], 32, 3, 1, 1), (2, 16, 8, 80, [700, 333], 32, 3, 1, 1), (2, 8, 4, 100, [900, 640], 32, 20, 1, 1), (16, 16, 8, 1, [2600 - 17 * i for i in range(16)], 64, 32, 1, 2)])
def test_waves_and_chunks(B, Hq, Hkv, n, N_of, page, top, first, recent, dtype):
    q, k, v, bounds, table = _make(n, B, Hq, Hkv, n, N_of, page, dtype)
    cache = binding.Pages(k, v, table, bounds)
    blocks = select(cache, q, max(N_of), top, first, recent, None, N_of)
    out = attend(cache, q, blocks, max(N_of), None, N_of)
    for i in sorted({0, n // 2, n - 1}):               # (a row's list is its own)
        one = blocks[:, :, i:i + 1]
        N_then = [N - n + 1 + i for N in N_of]
        exact, tol = reference(q[:, :, i:i + 1], k, v, table, [1] * B, N_then, SCALE, _seen(one, page, N_then))
        compare(out[:, :, i:i + 1], exact, tol, [1] * B)
