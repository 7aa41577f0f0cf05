"""specache_block_select for more rows than go in one launch, by scratch memory or by number: the lists are those of its parts."""
import ctypes as C

import pytest
import torch

from paper_2503_16163_amd import binding
from paper_2503_16163_amd.binding import BlockConfig
from tests.paged import generator
from tests.test_gpu_blocks import lists, select
from tests.test_paged import _pages, _ref

GIB = 1 << 30


@pytest.mark.parametrize("batch,heads,group,tokens,kv_tokens,page", [
    (1, 8, 8, 32768, 131072, 16), (1, 32, 1, 32768, 131072, 16), (8, 8, 4, 512, 131072, 16), (2, 8, 3, 1499, 131072, 16), (1, 1, 1, 131072, 1 << 22, 16), (4, 32, 1, 32767, 4096, 256)])
def test_scratch_memory_is_bounded(batch, heads, group, tokens, kv_tokens, page):
    size = C.c_int64()
    cache = _pages(n_kv_heads=heads, page_tokens=page, table_pages=kv_tokens // page)
    assert binding.lib().specache_block_scratch(_ref(cache), _ref(BlockConfig(batch, heads * group, tokens, kv_tokens, 16, 1, 1, 0.0)), C.byref(size)) == binding.OK
    assert 0 < size.value <= GIB


def test_one_launch_s_rows_of_the_longest_context():
    """Tokens whose heads make one product's rows stay together: up to 16, of 2^24 blocks each."""
    size = C.c_int64()
    assert binding.lib().specache_block_scratch(_ref(_pages(n_kv_heads=1, table_pages=1 << 24)), _ref(BlockConfig(1, 1, 4096, 1 << 28, 16, 1, 1, 0.0)), C.byref(size)) == binding.OK
    assert size.value == 16 * (1 << 24) * 12.25


def test_most_lists():
    size = C.c_int64()
    cache = _pages(n_kv_heads=1)
    for tokens, want in (((1 << 22) - 1, binding.OK), (1 << 22, binding.EINVAL)):
        cfg = BlockConfig(1, 2, tokens, 160, 3, 1, 1, 0.0)
        assert binding.lib().specache_block_scratch(_ref(cache), _ref(cfg), C.byref(size)) == want
    q, lists_at = binding.View(1 << 20, 1 << 40, 1 << 30, 128), 1 << 20
    assert binding.lib().specache_block_select(_ref(cache), _ref(cfg), _ref(q), lists_at, None, None, lists_at, 1 << 40, None) == binding.EINVAL


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("Hq,Hkv,n,n_of,N_of,page,alike", [
    (32, 8, 1500, [1500, 700], [131072, 100001], 16, False), (9, 3, 4999, [4999, 4998], [131072, 131071], 16, False), (8, 8, 2500, [2500, 2500], [70000, 131072], 16, False),
    (8, 2, 6500, [6500, 6400], [131072, 100000], 16, True)])     # (all scores alike: told apart in 64 bits in the scratch memory)
def test_slices(Hq, Hkv, n, n_of, N_of, page, alike, dtype):
    B, most, top, first, recent = 2, 131072, 20, 1, 2
    gen = generator(n)
    P = most // page + 3
    bounds = torch.randn((P, Hkv, 2, 128), generator=gen, device="cuda").to(dtype)
    bounds = torch.stack([bounds.amin(dim=2), bounds.amax(dim=2)], dim=2)
    if alike:
        bounds[:] = bounds[:1].clone()
    table = torch.stack([torch.randperm(P, generator=gen, device="cuda")[:most // page] for _ in range(B)]).to(torch.int32)
    table[1, 77] = -1
    k = torch.zeros((1, Hkv, page, 128), dtype=dtype, device="cuda").expand(P, Hkv, page, 128)     # (not read)
    q = torch.randn((B, Hq, n, 128), generator=gen, device="cuda").to(dtype)
    cache = binding.Pages(k, k, table, bounds)
    blocks = 12.25 * most // page
    assert binding.block_scratch(cache, B, Hq, n, most, top, first, recent) < B * Hkv * n * blocks / 2, "these are not several slices"
    got = select(cache, q, most, top, first, recent, n_of, N_of)
    for b in range(B):
        assert bool((got[b, :, n_of[b]:] == -9).all())
        # by parts that go in one launch
        alone = binding.Pages(k, k, table[b:b + 1], bounds)
        step = 100
        assert binding.block_scratch(alone, 1, Hq, step, most, top, first, recent) == Hkv * step * blocks
        for i in range(0, n_of[b], step):
            m = min(step, n_of[b] - i)
            part = select(alone, q[b:b + 1, :, i:i + m], most, top, first, recent, None, [N_of[b] - n_of[b] + i + m])
            assert torch.equal(part[0], got[b, :, i:i + m])
        for i in (0, n_of[b] // 2, n_of[b] - 1):
            want = lists(q[b:b + 1, :, i:i + 1], bounds, table[b:b + 1], [1], [N_of[b] - n_of[b] + i + 1], page, top, first, recent)
            assert torch.equal(want[0], got[b, :, i:i + 1])


@pytest.mark.gpu
def test_more_rows_than_a_launch_has_workgroups():
    """Prompts of 66000 tokens for 32 heads, the first block and the rows' own; then a few blocks to choose from."""
    Hkv, n, page = 32, 66000, 256
    gen = generator(1)
    width = -(-n // page)
    k = torch.zeros((1, Hkv, page, 128), dtype=torch.float16, device="cuda").expand(width, Hkv, page, 128)
    table = torch.arange(width, dtype=torch.int32, device="cuda")[None]
    # a block's bounds are alike in all channels: of queries that are positive the best blocks are those of the largest bounds
    level = torch.randperm(width, generator=gen, device="cuda")
    bounds = level.to(torch.float16)[:, None, None, None].expand(width, Hkv, 2, 128).contiguous()
    q = torch.rand((1, 1, n, 128), generator=gen, device="cuda").add_(0.5).to(torch.float16).expand(1, Hkv, n, 128)
    cache = binding.Pages(k, k, table, bounds)
    mine = torch.arange(n, device="cuda") // page
    got = select(cache, q, n, 0, 1, 1)
    want = torch.stack([torch.zeros_like(mine), torch.where(mine > 0, mine, -1)], dim=1).to(torch.int32)
    assert bool((got == want).all())
    got = select(cache, q, n, 2, 0, 0)
    seen = torch.where(torch.arange(width, device="cuda") <= mine[:, None], level, -1)
    value, index = seen.topk(2, dim=1)
    index = torch.where(value >= 0, index, width).sort(dim=1)[0]
    assert bool((got == torch.where(index < width, index, -1).to(torch.int32)).all())
