"""specache_paged_append of more tokens than one launch has workgroups for, up to the 2^30 that its description names."""
import pytest
import torch

from paper_2503_16163_amd import binding
from tests.paged import generator, ints

pytestmark = pytest.mark.gpu


def _turned(plan, x, at):
    """x [n, 128] at positions at [n]."""
    out = torch.empty((1, 1, len(at), 128), dtype=x.dtype, device="cuda")
    binding.rotate(plan, x[None, None].contiguous(), out, positions=at.to(torch.int32)[None].contiguous())
    return out[0, 0]


def test_a_step_of_many_sequences():
    """2^23 + 5 sequences take a step; a few hundred of them, the first and the last among them, have a page."""
    B, page, gen = (1 << 23) + 5, 16, generator(1)
    x = torch.randn((B, 1, 1, 128), generator=gen, device="cuda", dtype=torch.bfloat16)
    out = torch.full_like(x, 7.0)
    have = torch.cat([torch.arange(100), (1 << 22) + torch.arange(-50, 50), B - 100 + torch.arange(100)]).cuda()
    k = torch.full((300, 1, page, 128), 7.0, device="cuda", dtype=torch.bfloat16)
    v, bounds = k.clone(), torch.full((300, 1, 2, 128), 7.0, device="cuda", dtype=torch.bfloat16)
    table = torch.full((B, 1), -1, dtype=torch.int32, device="cuda")
    table[have, 0] = torch.arange(300, dtype=torch.int32, device="cuda")
    starts = torch.randint(0, page, (B,), generator=gen, device="cuda", dtype=torch.int32)
    at = torch.randint(0, 1 << 20, (B, 1), generator=gen, device="cuda", dtype=torch.int32)
    plan = binding.rotary_plan()
    binding.paged_append(binding.Pages(k, v, table, bounds), plan, x, x, x, out, starts, positions=at)
    want = torch.empty_like(out)
    binding.rotate(plan, x, want, positions=at)
    assert torch.equal(out, want)
    want_k, want_v, want_bounds, i, s = torch.full_like(k, 7.0), torch.full_like(v, 7.0), torch.full_like(bounds, 7.0), torch.arange(300, device="cuda"), starts[have].long()
    want_k[i, 0, s], want_v[i, 0, s] = out[have, 0, 0], x[have, 0, 0]
    fresh = (s == 0)[:, None]
    want_bounds[:, 0, 0] = torch.where(fresh, out[have, 0, 0], out[have, 0, 0].clamp(max=7.0))
    want_bounds[:, 0, 1] = torch.where(fresh, out[have, 0, 0], out[have, 0, 0].clamp(min=7.0))
    assert torch.equal(k, want_k) and torch.equal(v, want_v) and torch.equal(bounds, want_bounds)


@pytest.mark.parametrize("with_bounds", [False, True])
def test_a_prompt_of_many_pages(with_bounds):
    """2^27 + 100 tokens (one row again and again) behind 5 others, pages of 16, of which a few are there."""
    n, page, start, gen = (1 << 27) + 100, 16, 5, generator(2)
    row = torch.randn(128, generator=gen, device="cuda", dtype=torch.float16)
    x = row.expand(1, 1, n, 128)
    width = -(-(start + n) // page)
    have = torch.cat([torch.arange(40), (1 << 22) + torch.arange(-20, 20), (1 << 23) + torch.arange(-20, 0), torch.arange(width - 6, width)]).cuda()
    P = len(have)
    k = torch.full((P, 1, page, 128), 7.0, device="cuda", dtype=torch.float16)
    v, bounds = k.clone(), torch.full((P, 1, 2, 128), 7.0, device="cuda", dtype=torch.float16)
    table = torch.full((1, width), -1, dtype=torch.int32, device="cuda")
    table[0, have] = torch.arange(P, dtype=torch.int32, device="cuda")
    plan = binding.rotary_plan(64)
    binding.paged_append(binding.Pages(k, v, table, bounds if with_bounds else None), plan, x, x, starts=ints([start]))
    at = have[:, None] * page + torch.arange(page, device="cuda")
    there = ((at >= start) & (at < start + n))[..., None]
    turned = _turned(plan, row.expand(P * page, 128), at.flatten()).view(P, page, 128)
    assert torch.equal(k[:, 0], torch.where(there, turned, 7.0)) and torch.equal(v[:, 0], torch.where(there, row, 7.0))
    low, high = torch.where(there, turned, torch.inf).amin(dim=1), torch.where(there, turned, -torch.inf).amax(dim=1)
    low[0], high[0] = low[0].clamp(max=7.0), high[0].clamp(min=7.0)     # (its place 0 was there before)
    if with_bounds:
        assert torch.equal(bounds[:, 0, 0], low) and torch.equal(bounds[:, 0, 1], high)
    else:
        assert bool((bounds == 7.0).all())


def test_the_queries_of_many_tokens():
    """2^25 + 3 tokens of a head, four to a workgroup: the queries alone come to more than a launch."""
    n, gen = (1 << 25) + 3, generator(3)
    x = torch.randn((1, 1, n, 128), generator=gen, device="cuda", dtype=torch.float16)
    out = torch.full_like(x, 7.0)
    k = torch.full((1, 1, 256, 128), 7.0, device="cuda", dtype=torch.float16)
    table = torch.full((1, -(-n // 256)), -1, dtype=torch.int32, device="cuda")
    table[0, -1] = 0
    binding.paged_append(binding.Pages(k, k.clone(), table), None, x, x, x, out)
    assert torch.equal(out, x)
    last = n - (table.shape[1] - 1) * 256
    assert torch.equal(k[0, 0, :last], x[0, 0, -last:]) and bool((k[0, 0, last:] == 7.0).all())
