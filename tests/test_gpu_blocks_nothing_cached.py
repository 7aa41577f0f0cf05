"""specache_block_attend where nothing is cached, and lists that name blocks all the same: those are no blocks of the sequence's tokens, and the rows give zeros."""
import ctypes as C

import pytest
import torch

from paper_2503_16163_amd import binding
from tests.paged import compare, generator, ints, reference, scratch_of
from tests.test_gpu_blocks import SCALE, _make, _seen, attend

pytestmark = pytest.mark.gpu
TYPES = [torch.float16, torch.bfloat16]


def _naming(B, Hkv, n, slots):
    """Lists of blocks 0, 1, ..: as many as there are entries."""
    return torch.arange(slots, dtype=torch.int32, device="cuda").expand(B, Hkv, n, slots).contiguous()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,slots,kv_tokens", [(1, 3, 160), (2, 3, 0), (1, 64, 1024), (40, 5, 80)])     # (64 entries: joined by a merge)
def test_a_cache_of_no_pages(n, slots, kv_tokens, dtype):
    B, Hq, Hkv, page = 2, 8, 2, 16
    k = torch.empty((0, Hkv, page, 128), dtype=dtype, device="cuda")
    table = torch.zeros((B, 64), dtype=torch.int32, device="cuda")
    q = torch.randn((B, Hq, n, 128), generator=generator(1), device="cuda").to(dtype)
    cache = binding.Pages(k, k, table)
    assert bool((attend(cache, q, _naming(B, Hkv, n, slots), kv_tokens) == 0).all())
    assert bool((attend(cache, q, _naming(B, Hkv, n, slots), kv_tokens, None, [kv_tokens, 0]) == 0).all())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,slots", [(1, 3), (3, 70)])
def test_no_cached_tokens_and_no_memory_behind_the_pages(n, slots, dtype):
    """kv_tokens = 0: the views and the table are asked for nothing."""
    B, Hq, Hkv, page = 2, 8, 2, 16
    q = torch.randn((B, Hq, n, 128), generator=generator(2), device="cuda").to(dtype)
    out, blocks = torch.full_like(q, 7.0), _naming(B, Hkv, n, slots)
    nowhere = binding.View(None, 0, 0, 0)
    cache = binding.PagesConfig(nowhere, nowhere, nowhere, None, 0, 5, Hkv, page, 0, 128, binding.FP16 if dtype == torch.float16 else binding.BF16)
    cfg, need, L = binding.BlockConfig(B, Hq, n, 0, slots, 0, 0, 0.0), C.c_int64(), binding.lib()
    assert L.specache_block_scratch(C.addressof(cache), C.addressof(cfg), C.byref(need)) == binding.OK
    scratch = scratch_of(need.value)
    views = [binding.View(x.data_ptr(), x.stride(0), x.stride(1), x.stride(2)) for x in (q, out)]
    assert L.specache_block_attend(C.addressof(cache), C.addressof(cfg), C.byref(views[0]), C.byref(views[1]), blocks.data_ptr(), None, None,
                                   scratch.data_ptr() if need.value else None, need.value, torch.cuda.current_stream().cuda_stream) == binding.OK
    assert bool((out == 0).all())


@pytest.mark.parametrize("dtype", TYPES)
def test_sequences_without_tokens_beside_others(dtype):
    N_of = [0, 200, 0, 16]
    q, k, v, bounds, table = _make(3, 4, 8, 2, 2, [200] * 4, 16, dtype)
    cache = binding.Pages(k, v, table)
    blocks = _naming(4, 2, 2, 7)
    got = attend(cache, q, blocks, 200, None, N_of)
    assert bool((got[0] == 0).all()) and bool((got[2] == 0).all())
    exact, tol = reference(q, k, v, table, [2] * 4, N_of, SCALE, _seen(blocks, 16, N_of))
    compare(got, exact, tol, [2] * 4)
