"""Counts that do not fit 32 bits are refused by the bindings of the paged calls, the scratch functions among them, and not cut off."""
import ctypes as C

import pytest

from paper_2503_16163_amd import binding
from paper_2503_16163_amd.binding import BlockConfig, PagedConfig
from tests.test_paged import _pages, _ref


class _Cache:
    def __init__(self, **change):
        self.config = _pages(**change)
        self.at = C.addressof(self.config)


WIDE = (2 ** 31, 2 ** 32 + 5, -2 ** 31 - 1, 2.0, None)


@pytest.mark.parametrize("wide", WIDE)
def test_scratch_functions_refuse(wide):
    cache = _Cache()
    counts = dict(batch=2, n_q_heads=4, q_tokens=3, kv_tokens=160)
    for call, more in ((binding.paged_scratch, dict(shared_tokens=0)), (binding.block_scratch, dict(top=3, first=1, recent=1))):
        assert call(cache, **counts, **more) >= 0
        for name in (*counts, *more):
            with pytest.raises(binding.SpeCacheError) as e:
                call(cache, **{**counts, **more, name: wide})
            assert e.value.code == binding.EINVAL


def test_scratch_functions_ask_for_what_the_library_says():
    size = C.c_int64()
    cache = _Cache(n_kv_heads=4, table_pages=2000)
    for counts in ((32, 4, 3, 20000, 16384), (1, 8, 1, 32000, 0), (2, 4, 1, 32000, 0)):
        assert binding.lib().specache_paged_scratch(_ref(cache.config), _ref(PagedConfig(*counts, 0.0)), C.byref(size)) == binding.OK
        assert binding.paged_scratch(cache, *counts) == size.value > 0
    for counts in ((2, 8, 3, 32000, 7, 1, 2), (1, 4, 1, 32000, 0, 900, 900)):
        assert binding.lib().specache_block_scratch(_ref(cache.config), _ref(BlockConfig(*counts, 0.0)), C.byref(size)) == binding.OK
        assert binding.block_scratch(cache, *counts) == size.value > 0


def test_tensors_of_more(monkeypatch):
    """By views that repeat one row: no memory of that size is behind them."""
    import torch
    binding._with_torch()
    monkeypatch.setattr(binding, "_here", lambda: -1)
    x, table = torch.zeros((1, 1, 16, 128), dtype=torch.float16), torch.zeros((1, 2), dtype=torch.int32)
    cache = binding.Pages(x, x, table)
    far = 2 ** 32 + 1
    tokens, heads, few = x[:, :, :1].expand(1, 1, far, 128), x[:, :, :1].expand(1, far, 1, 128), x[:, :, :1]
    pages, wide = x.expand(far, 1, 16, 128), x[:, :, :1].expand(1, 1, 2 ** 32 + 16, 128)
    for make in (lambda: binding.paged_append(cache, None, tokens, tokens), lambda: binding.paged_append(cache, None, few, few, heads, heads),
                 lambda: binding.paged_attend(cache, heads, heads), lambda: binding.block_attend(cache, tokens, tokens, torch.zeros((1, 1, 1, 1), dtype=torch.int32).expand(1, 1, far, 1)),
                 lambda: binding.Pages(pages, pages, table), lambda: binding.Pages(wide, wide, table)):
        with pytest.raises(binding.SpeCacheError) as e:
            make()
        assert e.value.code == binding.EINVAL
