"""Many sequences, or many lists, over many positions: splitting their walks never makes a call that is refused, nor takes more than some GiB of scratch memory."""
import ctypes as C

import pytest
import torch

from paper_2503_16163_amd import binding
from paper_2503_16163_amd.binding import BlockConfig, PagedConfig
from tests.paged import attend, compare, generator, pool, reference
from tests.test_paged import _pages, _ref

GIB = 1 << 30


@pytest.mark.parametrize("batch,heads,kv_tokens", [(2048, 32, 131072), (8192, 8, 131072), (65535, 8, 1 << 22), (1 << 21, 1, 1 << 20), ((1 << 22) - 1, 1, 1 << 20)])
def test_many_steps(batch, heads, kv_tokens):
    size = C.c_int64()
    cache = _pages(n_kv_heads=heads, table_pages=kv_tokens // 16)
    for group in (1, 4, 64):
        if batch * heads * group > 1 << 28:
            continue
        for shared in (0, kv_tokens):
            assert binding.lib().specache_paged_scratch(_ref(cache), _ref(PagedConfig(batch, heads * group, 1, kv_tokens, shared, 0.0)), C.byref(size)) == binding.OK, (group, shared)
            assert size.value <= GIB if not shared else 3 * GIB


@pytest.mark.parametrize("tokens,heads,entries", [(32768, 32, 256), (32768, 8, 4096), (65535, 32, 1 << 16), (4096, 8, 1024)])
def test_many_long_lists(tokens, heads, entries):
    size = C.c_int64()
    cache = _pages(n_kv_heads=heads, table_pages=1 << 16, page_tokens=64)
    for group in (1, 8):
        assert binding.lib().specache_block_scratch(_ref(cache), _ref(BlockConfig(1, heads * group, tokens, 1 << 22, 0, entries, 0, 0.0)), C.byref(size)) == binding.OK, group
        assert size.value <= GIB


@pytest.mark.parametrize("heads,group,tokens", [(1, 1, 1), (8, 4, 8), (1, 4, 16), (32, 1, 1), (1, 1, 64), (2, 8, 16)])
def test_the_counts_that_specache_h_names(heads, group, tokens):
    """The most sequences that it promises are taken, one more than a launch has workgroups or than 2^28 rows is refused; partial results fit 4 GiB with a prefix that is shared."""
    size = C.c_int64()
    cache = _pages(n_kv_heads=heads, table_pages=1 << 16)
    most = min(((1 << 22) - 1) // (heads * -(-tokens * group // 128)), (1 << 28) // (heads * group * tokens))
    for batch, want in ((most, binding.OK), (most + 1, binding.EINVAL)):
        for kv_tokens, shared in ((1, 0), (1 << 20, 0), (1 << 20, 1 << 19), (1 << 20, 1 << 20)):
            size.value = 0
            assert binding.lib().specache_paged_scratch(_ref(cache), _ref(PagedConfig(batch, heads * group, tokens, kv_tokens, shared, 0.0)), C.byref(size)) == want, (batch, shared)
            assert size.value <= (4 * GIB if shared else GIB)
    for batch in (1000, 22705, 47727):
        if batch <= most:
            assert binding.lib().specache_paged_scratch(_ref(cache), _ref(PagedConfig(batch, heads * group, tokens, 1 << 20, 1 << 19, 0.0)), C.byref(size)) == binding.OK
            assert size.value <= 4 * GIB


@pytest.mark.gpu
def test_many_steps_of_few_pages():
    """2100 sequences and 32 heads of up to 131072 positions; most have a few, and all have their pages of one row of the table."""
    B, H, width, page = 2100, 32, 8192, 16
    gen = generator(5)
    k, v = pool(gen, 300, H, page, torch.bfloat16)
    table = torch.randint(0, 300, (1, width), generator=gen, device="cuda").to(torch.int32).expand(B, width)
    q = torch.randn((B, H, 1, 128), generator=gen, device="cuda").to(torch.bfloat16)
    N_of = [1 + 7 * b % 1000 for b in range(B)]
    N_of[3], N_of[700], N_of[2099], N_of[1500] = width * page, 9999, 70001, 0
    got = attend(binding.Pages(k, v, table), q, width * page, 0, None, N_of)
    for b in (0, 3, 5, 700, 1234, 1500, 2098, 2099):
        exact, tol = reference(q[b:b + 1, ::8], k[:, ::8], v[:, ::8], table[b:b + 1], [1], [N_of[b]], 128 ** -0.5)
        compare(got[b:b + 1, ::8], exact, tol, [1])
