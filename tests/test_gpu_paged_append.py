"""specache_paged_append against the formulas in 64 bits: queries and keys within the rounding of specache_rotate's tests, values and bounds exactly, everything
else as it was."""
import math

import pytest
import torch

from paper_2503_16163_amd import binding
from tests.paged import generator, ints, pool, table_of
from tests.test_gpu_rotary import _bound, _expected
from tests.test_operators import _frequencies

pytestmark = pytest.mark.gpu


def _case(seed, B, L, Hq, Hkv, page, dtype, order="heads", starts=None, lengths=None, width=None):
    gen = generator(seed)
    x = torch.randn((B, L, Hq + 2 * Hkv, 128), generator=gen, device="cuda").to(dtype).transpose(1, 2)
    ends = [max(a + n, 0) for a, n in zip(starts or [0] * B, lengths or [L] * B)]
    width = max(1, -(-max(ends) // page)) if width is None else width
    table, pages = table_of(gen, [min(e, width * page) for e in ends], page, width)
    k, v = pool(gen, pages, Hkv, page, dtype, order, fill=False)
    bounds = torch.randn((pages, Hkv, 2, 128), generator=gen, device="cuda").to(dtype)
    return x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:], k, v, bounds, table


def _expect(k_turned, v_new, k, v, bounds, table, starts, lengths):
    """The pages and bounds after the rounded keys and the values went in, token by token's place."""
    k, v, bounds = k.clone(), v.clone(), bounds.clone()
    P, H, T, _ = k.shape
    row = table.tolist()
    for b, (start, n) in enumerate(zip(starts, lengths)):
        first = max(start, 0)
        for i in range(first // T, (start + n - 1) // T + 1 if start + n > first else 0):
            if i >= len(row[b]) or not 0 <= row[b][i] < P:
                continue
            lo, hi, page = max(first, i * T), min(start + n, i * T + T), row[b][i]
            keys = k_turned[b, :, lo - start:hi - start]
            k[page, :, lo - i * T:hi - i * T] = keys
            v[page, :, lo - i * T:hi - i * T] = v_new[b, :, lo - start:hi - start]
            low, high = keys.float().nan_to_num(math.inf, math.inf, -math.inf).amin(dim=1), keys.float().nan_to_num(-math.inf, math.inf, -math.inf).amax(dim=1)
            if lo > i * T:
                low, high = torch.minimum(low, bounds[page, :, 0].float()), torch.maximum(high, bounds[page, :, 1].float())
            bounds[page, :, 0], bounds[page, :, 1] = low.to(k.dtype), high.to(k.dtype)
    return k, v, bounds


def _check(case, plan, starts=None, lengths=None, positions=None, with_bounds=True, f=None):
    q, k_new, v_new, k, v, bounds, table = case
    B, Hq, L, _ = q.shape
    q_out = torch.full(q.shape, 7.0, device="cuda", dtype=q.dtype)
    before = (k.clone(), v.clone(), bounds.clone())
    cache = binding.Pages(k, v, table, bounds if with_bounds else None)
    binding.paged_append(cache, plan, k_new, v_new, q, q_out, ints(starts), ints(lengths), None if positions is None else positions)
    s, n = starts or [0] * B, [min(max(x, 0), L) for x in lengths] if lengths else [L] * B
    at = positions if positions is not None else ints(s)[:, None] + torch.arange(L, device="cuda", dtype=torch.int32)
    asked = torch.arange(L, device="cuda")[None] < ints(n)[:, None]
    # the keys' rounding is the rotation's own
    turned = torch.empty_like(k_new.contiguous())
    if plan is None:
        assert torch.equal(q_out.transpose(1, 2)[asked], q.transpose(1, 2)[asked])
        turned.copy_(k_new)
    else:
        binding.rotate(plan, k_new, turned, positions=at.contiguous())
        if f is not None:
            for y, t in ((q_out, q), (turned, k_new)):
                e = _expected(t, at, f, plan.gain, plan.rotary_dim, plan.layout)
                d = plan.rotary_dim
                off = ((y.double() - e).abs() - _bound(e, t.double(), plan.gain, q.dtype, d, plan.layout))[..., :d]
                assert bool((off.transpose(1, 2)[asked] <= 0).all())
                assert torch.equal(y.transpose(1, 2)[asked][..., d:], t.transpose(1, 2)[asked][..., d:])
    assert bool((q_out.transpose(1, 2)[~asked] == 7.0).all())
    want_k, want_v, want_bounds = _expect(turned, v_new, *before, table, s, n)
    assert torch.equal(k.nan_to_num(1e4), want_k.nan_to_num(1e4)) and torch.equal(v, want_v)
    assert torch.equal(bounds, want_bounds if with_bounds else before[2])
    return cache


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("layout", [0, 1])
@pytest.mark.parametrize("B,L,Hq,Hkv,d,scaling,page,starts", [
    (1, 1, 1, 1, 128, 0, 16, None), (1, 2, 32, 8, 128, 3, 64, [63]), (3, 5, 5, 5, 64, 1, 16, [0, 14, 31]), (16, 1, 32, 8, 128, 0, 64, [37 * i for i in range(16)]),
    (2, 33, 8, 1, 96, 0, 32, [1, 95]), (1, 1000, 16, 4, 16, 2, 256, None), (2, 257, 7, 7, 112, 0, 128, [100, 0]), (1, 4000, 4, 2, 128, 0, 16, [7]),
    (2, 300, 3, 40, 32, 0, 64, [5, 64])])
def test_paged_append(B, L, Hq, Hkv, d, scaling, page, starts, layout, dtype):
    plan = binding.rotary_plan(d, 1.0e4, layout, scaling, 8.0, 4096, 1.0, 4.0)
    f = _frequencies(d, 1.0e4, scaling, 8.0, 4096, 1.0, 4.0)
    case = _case(B * 1000 + L, B, L, Hq, Hkv, page, dtype, "places" if L % 2 else "heads", starts)
    _check(case, plan, starts, f=f, with_bounds=d != 64)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("L,page,starts,lengths", [
    (1, 16, [5, 16, 100, 0], [1, 0, 1, 7]), (40, 16, [5, 16, 100, 0], [40, 0, 1, -3]), (300, 64, [0, 1, 63, 64], [300, 299, 1, 65]),
    (20, 32, [-5, -30, 90, 200], [20, 20, 20, 20]), (3, 16, [2 ** 31 - 2, -(2 ** 31), 14, 15], [3, 3, 3, 3])])
def test_ragged_batches_and_positions_without_a_place(L, page, starts, lengths, dtype):
    """Sequences without tokens, positions before the first, behind the table or where it names no page: nothing of them is written."""
    width = 8
    case = _case(L + page, 4, L, 4, 2, page, dtype, "heads", [0] * 4, [width * page] * 4, width)
    table = case[6]
    table[2, 6] = -1
    table[3, 7] = case[3].shape[0]
    table[1, 0] = 2 ** 31 - 1
    q, k_new, v_new = case[:3]
    for b in range(4):
        n = min(max(lengths[b], 0), L)
        for x in (q, k_new, v_new):
            x[b, :, n:] = math.nan
    starts_t = starts
    plan = binding.rotary_plan()
    q_out = torch.full(q.shape, 7.0, device="cuda", dtype=dtype)
    if max(abs(s) for s in starts) < 2 ** 20:
        _check(case, plan, starts_t, lengths, f=_frequencies(128, 1.0e4, 0, 1.0, 0, 0, 0))
    else:                                   # (positions of the rotation given: those of the far tokens pass 32 bits)
        at = torch.arange(4 * L, device="cuda", dtype=torch.int32).view(4, L)
        _check(case, plan, starts_t, lengths, positions=at)


def test_without_a_plan_and_without_queries():
    for dtype in (torch.float16, torch.bfloat16):
        case = _case(3, 2, 50, 4, 2, 16, dtype, starts=[3, 0])
        _check(case, None, [3, 0])
        q, k_new, v_new, k, v, bounds, table = _case(3, 2, 50, 4, 2, 16, dtype, starts=[3, 0])
        binding.paged_append(binding.Pages(k, v, table, bounds), None, k_new, v_new, starts=ints([3, 0]))
        assert torch.equal(k, case[3]) and torch.equal(v, case[4]) and torch.equal(bounds, case[5])


def test_nan_keys_are_passed_over_by_the_bounds():
    case = _case(8, 1, 40, 2, 2, 16, torch.bfloat16)
    case[1][0, 0, 5, 3] = math.nan
    case[1][0, 1, 20:36, 9] = math.nan
    case[1][0, 1, 2, 9] = math.inf
    cache = _check(case, None)
    page = case[6][0, 0].item()
    assert bool(torch.isfinite(case[5][page, 0].float()).all()) and torch.isinf(case[5][page, 1, 1, 9])


def test_token_by_token_is_all_at_once():
    """A prompt, then its tokens one and two at a time: the same pages and bounds; queries in place."""
    plan = binding.rotary_plan(64, layout=binding.ROTARY_INTERLEAVED)
    B, L = 2, 70
    q, k_new, v_new, k, v, bounds, table = _case(9, B, L, 4, 2, 32, torch.float16)
    whole = tuple(torch.zeros_like(x) for x in (k, v, bounds))
    parts = tuple(torch.zeros_like(x) for x in (k, v, bounds))
    q_out = torch.empty_like(q)
    binding.paged_append(binding.Pages(whole[0], whole[1], table, whole[2]), plan, k_new, v_new, q, q_out)
    cache, t = binding.Pages(parts[0], parts[1], table, parts[2]), 0
    mine = q.clone()
    for n in [1, 2, 1, 30, 1, 1, 2, 2, 1, 29]:
        here = slice(t, t + n)
        binding.paged_append(cache, plan, k_new[:, :, here], v_new[:, :, here], mine[:, :, here], mine[:, :, here], starts=ints([t] * B))
        t += n
    assert t == L and torch.equal(mine, q_out)
    for a, b in zip(whole, parts):
        assert torch.equal(a, b)


def test_large_prompts_and_far_pages():
    """Stores past the caches, pages whose offsets pass 32 bits."""
    flat = torch.zeros(5 << 30, device="cuda", dtype=torch.float16)
    case = list(_case(10, 1, 2400, 32, 8, 64, torch.float16, starts=[17]))
    far = flat.as_strided((40, 8, 64, 128), (1 << 27, 64 * 128, 128, 1))
    assert case[3].shape[0] <= 41
    case[6] = torch.where(case[6] >= 40, -1, case[6])
    case[3], case[4], case[5] = far, case[4][:40].contiguous(), case[5][:40].contiguous()
    q, k_new, v_new, k, v, bounds, table = case
    near = torch.zeros_like(v)
    plan = binding.rotary_plan()
    a, b = torch.empty_like(q), torch.empty_like(q)
    binding.paged_append(binding.Pages(near, v, table), plan, k_new, v_new, q, a, ints([17]))
    binding.paged_append(binding.Pages(k, v, table), plan, k_new, v_new, q, b, ints([17]))
    assert torch.equal(a, b) and torch.equal(k, near)
    del flat, far, k, case
    case = _case(11, 3, 9000, 32, 8, 16, torch.bfloat16, starts=[0, 5, 16])
    _check(case, binding.rotary_plan(128, 5.0e5), [0, 5, 16], f=_frequencies(128, 5.0e5, 0, 1.0, 0, 0, 0))


def test_captured_while_positions_move():
    plan = binding.rotary_plan()
    q, k_new, v_new, k, v, bounds, table = _case(12, 4, 2, 8, 2, 16, torch.bfloat16, lengths=[200] * 4)
    x = torch.empty_like(q)
    mine = tuple(torch.zeros_like(t) for t in (k, v, bounds))
    want = tuple(torch.zeros_like(t) for t in (k, v, bounds))
    starts = torch.zeros(4, dtype=torch.int32, device="cuda")
    cache, plain = binding.Pages(mine[0], mine[1], table, mine[2]), binding.Pages(want[0], want[1], table, want[2])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        binding.paged_append(cache, plan, k_new, v_new, q, x, starts)
    for turn in range(4):
        k_new.copy_(torch.randn_like(k_new))
        starts.copy_(ints([7 * turn, 2 * turn, 50 + turn, 16 * turn]))
        y = torch.empty_like(q)
        binding.paged_append(plain, plan, k_new, v_new, q, y, starts)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(x, y) and all(torch.equal(a, b) for a, b in zip(mine, want))


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("with_bounds", [False, True])
@pytest.mark.parametrize("layout,d", [(0, 128), (0, 96), (1, 128), (1, 64)])
def test_more_than_the_caches_hold(layout, d, with_bounds, dtype):
    """Prompts whose stores go past the caches (from 32 MiB on), ragged, from inside a page on."""
    plan = binding.rotary_plan(d, 1.0e4, layout)
    starts, lengths = [37, 300], [6000, 5555]
    case = _case(d + layout, 2, 6000, 8, 2, 128, dtype, "places" if layout else "heads", starts, lengths)
    _check(case, plan, starts, lengths, with_bounds=with_bounds, f=_frequencies(d, 1.0e4, 0, 1.0, 0, 0, 0))


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("layout,d", [(0, 128), (0, 96), (1, 128)])
def test_small_calls_without_bounds(layout, d, dtype):
    case = _case(d, 3, 9, 4, 2, 16, dtype, "heads", [3, 15, 16])
    _check(case, binding.rotary_plan(d, 1.0e4, layout), [3, 15, 16], with_bounds=False, f=_frequencies(d, 1.0e4, 0, 1.0, 0, 0, 0))
