"""What the calls on a paged cache refuse, on the CPU: every check here returns before any GPU call, and no pointer is followed."""
import ctypes as C
import math
import os
import re

import pytest

from paper_2503_16163_amd import binding
from paper_2503_16163_amd.binding import BlockConfig, PagedConfig, PagesConfig, Rotary, View

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
A = 1 << 20     # an address that nothing reads


@pytest.mark.parametrize("name,struct", [("specache_pages", PagesConfig), ("specache_paged_config", PagedConfig), ("specache_block_config", BlockConfig)])
def test_structs_match_header_field_order(name, struct):
    text = open(os.path.join(ROOT, "include", "specache.h")).read()
    body = re.search(r"typedef struct %s \{(.*?)\} %s;" % (name, name), text, flags=re.S).group(1)
    body = re.sub(r"/\*.*?\*/", "", body, flags=re.S)
    names = [n.strip(" *") for line in re.findall(r"\b(?:const int32_t\*|specache_view|u?int\d+_t|float)\s+([^;]*);", body) for n in line.split(",")]
    assert names == [f[0] for f in struct._fields_]
    assert C.sizeof(PagesConfig) == 3 * 32 + 16 + 24 and C.sizeof(PagedConfig) == 24 and C.sizeof(BlockConfig) == 32


def _pages(**change):
    c = PagesConfig(View(A, 4096, 2048, 128), View(2 * A, 4096, 2048, 128), View(3 * A, 512, 256, 128), A, 10, 8, 2, 16, 10, 128, 0)
    for k, v in change.items():
        setattr(c, k, v)
    return c


BAD_CACHES = [dict(n_pages=-1), dict(n_kv_heads=0), dict(page_tokens=8), dict(page_tokens=24), dict(page_tokens=512), dict(page_tokens=0), dict(table_pages=-1),
              dict(table_pages=(1 << 24) + 1), dict(head_dim=64), dict(dtype=2), dict(table_stride=-1)]
BAD_MEMORY = [dict(table=None), dict(table=A + 2), dict(k=View(None, 4096, 2048, 128)), dict(v=View(2 * A + 8, 4096, 2048, 128)), dict(k=View(A, 4096, -2048, 128)),
              dict(v=View(2 * A, 4096, 2048, 132)), dict(k=View(A, 4096, 2048, (1 << 20) + 8))]


def _ref(x):
    return None if x is None else C.byref(x)


def _append(cache, plan=None, batch=2, tokens=3, n_q=4, q=View(A, 1536, 384, 128), q_out=View(2 * A, 1536, 384, 128), k=View(A, 768, 384, 128),
            v=View(A, 768, 384, 128), starts=None, lengths=None, positions=None):
    return binding.lib().specache_paged_append(_ref(cache), _ref(plan), batch, tokens, n_q, _ref(q), _ref(q_out), _ref(k), _ref(v), starts, lengths, positions, None)


def test_append_refuses():
    for change in BAD_CACHES + BAD_MEMORY + [dict(bounds=View(3 * A + 2, 512, 256, 128)), dict(k=View(A, 0, 2048, 128)), dict(v=View(A, 4096, 2048, 0)),
                                             dict(bounds=View(3 * A, 512, 0, 128))]:
        assert _append(_pages(**change)) == binding.EINVAL, change
        assert binding.lib().specache_last_error(None)
    for change in (dict(plan=Rotary()), dict(batch=-1), dict(tokens=-1), dict(n_q=-1), dict(q=None), dict(q_out=None), dict(k=None), dict(v=None), dict(k=View(A + 4, 768, 384, 128)),
                   dict(v=View(A, 768, 380, 128)), dict(q_out=View(A, 1536, 128, 512)), dict(q_out=View(2 * A, 1536, 0, 128)), dict(starts=A + 1), dict(lengths=A + 2),
                   dict(positions=A + 3), dict(n_q=1 << 21), dict(batch=1 << 20, tokens=2048)):
        assert _append(_pages(), **change) == binding.EINVAL, change
    assert _append(None) == binding.EINVAL
    assert _append(_pages(), batch=0, k=None) == _append(_pages(), tokens=0, k=None) == binding.OK


def _attend(cache, cfg, q=View(A, 1536, 384, 128), out=View(4 * A, 1536, 384, 128), q_lengths=None, kv_lengths=None, scratch=None, size=0):
    return binding.lib().specache_paged_attend(_ref(cache), _ref(cfg), _ref(q), _ref(out), q_lengths, kv_lengths, scratch, size, None)


def _paged(**change):
    c = PagedConfig(2, 4, 3, 160, 0, 0.0)
    for k, v in change.items():
        setattr(c, k, v)
    return c


BAD_COUNTS = [dict(batch=-1), dict(q_tokens=-1), dict(kv_tokens=-1), dict(kv_tokens=161), dict(n_q_heads=3), dict(n_q_heads=0), dict(n_q_heads=130), dict(sm_scale=math.nan),
              dict(sm_scale=math.inf), dict(batch=1 << 15, q_tokens=1 << 14), dict(q_tokens=1 << 30)]
BAD_VIEWS = [dict(q=None), dict(out=None), dict(q=View(A + 2, 1536, 384, 128)), dict(out=View(4 * A, 1536, 0, 128)), dict(q=View(A, 1536, 384, 4)), dict(q_lengths=A + 1),
             dict(kv_lengths=A + 2)]


def test_attend_refuses():
    size = C.c_int64(-7)
    for change in BAD_CACHES:
        assert _attend(_pages(**change), _paged()) == binding.EINVAL, change
        assert binding.lib().specache_paged_scratch(_ref(_pages(**change)), _ref(_paged()), C.byref(size)) == binding.EINVAL
    for change in BAD_COUNTS + [dict(shared_tokens=-1)]:
        assert _attend(_pages(), _paged(**change)) == binding.EINVAL, change
        assert binding.lib().specache_paged_scratch(_ref(_pages()), _ref(_paged(**change)), C.byref(size)) == binding.EINVAL
    for change in BAD_MEMORY:
        assert _attend(_pages(**change), _paged()) == binding.EINVAL, change
    for views in BAD_VIEWS:
        assert _attend(_pages(), _paged(), **views) == binding.EINVAL, views
    assert size.value == -7
    assert _attend(None, _paged()) == _attend(_pages(), None) == binding.lib().specache_paged_scratch(_ref(_pages()), _ref(_paged()), None) == binding.EINVAL
    assert _attend(_pages(), _paged(batch=0), q=None) == _attend(_pages(), _paged(q_tokens=0), out=None) == binding.OK


def test_attend_wants_its_scratch_memory():
    size = C.c_int64()
    for cache, cfg in ((_pages(table_pages=10000), _paged(kv_tokens=100000)), (_pages(n_kv_heads=4, table_pages=2000), _paged(batch=32, kv_tokens=20000, shared_tokens=16384))):
        assert binding.lib().specache_paged_scratch(_ref(cache), _ref(cfg), C.byref(size)) == binding.OK and size.value > 0
        assert _attend(cache, cfg) == _attend(cache, cfg, scratch=A + 8, size=size.value) == binding.EINVAL
        assert _attend(cache, cfg, scratch=A, size=size.value - 1) == binding.ECAPACITY
    # what is shared counts in whole pages, for more than one sequence, and where it pays
    for cfg in (_paged(), _paged(shared_tokens=15), _paged(shared_tokens=32), _paged(batch=1, shared_tokens=160)):
        assert binding.lib().specache_paged_scratch(_ref(_pages()), _ref(cfg), C.byref(size)) == binding.OK and size.value == 0


def _block(**change):
    c = BlockConfig(2, 4, 3, 160, 3, 1, 1, 0.0)
    for k, v in change.items():
        setattr(c, k, v)
    return c


def _select(cache, cfg, q=View(A, 1536, 384, 128), blocks=A, q_lengths=None, kv_lengths=None, scratch=A, size=1 << 40):
    return binding.lib().specache_block_select(_ref(cache), _ref(cfg), _ref(q), blocks, q_lengths, kv_lengths, scratch, size, None)


def _block_attend(cache, cfg, q=View(A, 1536, 384, 128), out=View(4 * A, 1536, 384, 128), blocks=A, q_lengths=None, kv_lengths=None, scratch=A, size=1 << 40):
    return binding.lib().specache_block_attend(_ref(cache), _ref(cfg), _ref(q), _ref(out), blocks, q_lengths, kv_lengths, scratch, size, None)


def test_block_calls_refuse():
    size = C.c_int64(-7)
    for cache, cfg in [(_pages(**x), _block()) for x in BAD_CACHES] + [(_pages(), _block(**x)) for x in BAD_COUNTS] + \
                      [(_pages(), _block(**x)) for x in (dict(top=-1), dict(first=-1), dict(recent=-1), dict(top=0, first=0, recent=0), dict(top=1 << 20))]:
        assert _select(cache, cfg) == _block_attend(cache, cfg) == binding.lib().specache_block_scratch(_ref(cache), _ref(cfg), C.byref(size)) == binding.EINVAL
    assert size.value == -7
    for change in BAD_MEMORY[:2]:
        assert _select(_pages(**change), _block()) == _block_attend(_pages(**change), _block()) == binding.EINVAL, change
    for change in BAD_MEMORY[2:]:
        assert _block_attend(_pages(**change), _block()) == binding.EINVAL, change
    for bounds in (View(None, 512, 256, 128), View(3 * A + 2, 512, 256, 128), View(3 * A, 512, 256, 4)):
        assert _select(_pages(bounds=bounds), _block()) == binding.EINVAL
    for views in BAD_VIEWS:
        if "out" not in views:
            assert _select(_pages(), _block(), **views) == binding.EINVAL, views
        assert _block_attend(_pages(), _block(), **views) == binding.EINVAL, views
    for blocks in (None, A + 2):
        assert _select(_pages(), _block(), blocks=blocks) == _block_attend(_pages(), _block(), blocks=blocks) == binding.EINVAL
    assert binding.lib().specache_block_scratch(_ref(_pages()), _ref(_block()), C.byref(size)) == binding.OK and size.value > 0
    assert _select(_pages(), _block(), scratch=None) == _select(_pages(), _block(), scratch=A + 8) == binding.EINVAL
    assert _select(_pages(), _block(), size=size.value - 1) == binding.ECAPACITY
    for nothing in (dict(batch=0), dict(q_tokens=0)):
        assert _select(_pages(), _block(**nothing), q=None) == _block_attend(_pages(), _block(**nothing), q=None) == binding.OK
    assert _select(None, _block()) == _select(_pages(), None) == _block_attend(None, _block()) == _block_attend(_pages(), None) == binding.EINVAL


def test_bindings_refuse(monkeypatch):
    import torch
    binding._with_torch()
    x, table = torch.zeros((4, 2, 16, 128), dtype=torch.float16), torch.zeros((3, 2), dtype=torch.int32)
    q, blocks = torch.zeros((3, 4, 1, 128), dtype=torch.float16), torch.zeros((3, 2, 1, 5), dtype=torch.int32)
    new = torch.zeros((3, 2, 1, 128), dtype=torch.float16)
    monkeypatch.setattr(binding, "_here", lambda: -1)          # (get_device() of a host tensor)
    cache = binding.Pages(x, x, table)
    for make in (lambda: binding.Pages(x.float(), x.float(), table), lambda: binding.Pages(x, x[:2], table), lambda: binding.Pages(x, x, table.long()),
                 lambda: binding.Pages(x, x, torch.zeros((2, 3), dtype=torch.int32).t()), lambda: binding.Pages(x, x, table, x), lambda: binding.Pages(x[..., :64], x[..., :64], table),
                 lambda: binding.paged_append(cache, None, new, new, q), lambda: binding.paged_append(cache, None, new[:2], new[:2]),
                 lambda: binding.paged_append(cache, None, new.bfloat16(), new), lambda: binding.paged_append(cache, None, new, new, starts=torch.zeros(2, dtype=torch.int32)),
                 lambda: binding.paged_attend(cache, q[:2], q[:2]), lambda: binding.paged_attend(cache, q, q[:, :2]), lambda: binding.paged_attend(cache, q.float(), q.float()),
                 lambda: binding.block_select(cache, q, blocks, top=5), lambda: binding.block_attend(cache, q, q, blocks[..., :4]), lambda: binding.block_attend(cache, q, q, blocks[0]),
                 lambda: binding.block_attend(cache, q, q, blocks.long()), lambda: binding.paged_attend(cache, q, q, 2 ** 31), lambda: binding.paged_attend(cache, q, q, 32, -2 ** 40),
                 lambda: binding.block_attend(cache, q, q, blocks, 2 ** 33), lambda: binding.block_select(cache, q, blocks[..., :2].contiguous(), 32, 0, 2, 0.0)):
        with pytest.raises(binding.SpeCacheError) as e:
            make()
        assert e.value.code == binding.EINVAL
    monkeypatch.setattr(binding, "_here", lambda: 0)           # another device than the tensors'
    for make in (lambda: binding.Pages(x, x, table), lambda: binding.paged_attend(cache, q, q), lambda: binding.paged_append(cache, None, new, new),
                 lambda: binding.block_attend(cache, q, q, blocks)):
        with pytest.raises(binding.SpeCacheError) as e:
            make()
        assert e.value.code == binding.EINVAL


def test_the_current_stream_is_the_default(monkeypatch):
    import torch
    calls = []

    class Recorder:
        def __getattr__(self, name):
            return lambda *args: calls.append((name, args)) or binding.OK
    stream = type("Stream", (), {"cuda_stream": 0x5EED})
    binding._with_torch()
    monkeypatch.setattr(binding, "_here", lambda: -1)
    monkeypatch.setattr(binding, "lib", lambda: Recorder())
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: stream)
    x, table = torch.zeros((4, 2, 16, 128), dtype=torch.float16), torch.zeros((3, 2), dtype=torch.int32)
    q, blocks = torch.zeros((3, 4, 1, 128), dtype=torch.float16), torch.zeros((3, 2, 1, 5), dtype=torch.int32)
    cache = binding.Pages(x, x, table, torch.zeros((4, 2, 2, 128), dtype=torch.float16))
    for given, want in ((None, 0x5EED), (0, 0), (77, 77), (stream, 0x5EED)):
        del calls[:]
        binding.paged_append(cache, None, q[:, :2], q[:, :2], q, q, stream=given)
        binding.paged_attend(cache, q, q, stream=given)
        binding.block_select(cache, q, blocks, top=5, stream=given)
        binding.block_attend(cache, q, q, blocks, stream=given)
        assert [name for name, _ in calls] == ["specache_paged_append", "specache_paged_attend", "specache_block_select", "specache_block_attend"]
        assert all(args[-1] == want for _, args in calls)
