"""What the calls without a context refuse, and the worked-out rotary configurations, on the CPU: every check here returns before any
GPU call, and no pointer is followed."""
import ctypes as C
import math
import re
import os

import pytest

from paper_2503_16163_amd import binding
from paper_2503_16163_amd.binding import Rotary, RotaryConfig, SampleConfig, View, WindowConfig

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
A = 1 << 20     # an address that nothing reads


@pytest.mark.parametrize("name,struct", [("specache_view", View), ("specache_rotary_config", RotaryConfig), ("specache_rotary", Rotary),
                                         ("specache_window_config", WindowConfig), ("specache_sample_config", SampleConfig)])
def test_structs_match_header_field_order(name, struct):
    text = open(os.path.join(ROOT, "include", "specache.h")).read()
    body = re.search(r"typedef struct %s \{(.*?)\} %s;" % (name, name), text, flags=re.S).group(1)
    body = re.sub(r"/\*.*?\*/", "", body, flags=re.S)
    names = [n.strip(" *").split("[")[0] for line in re.findall(r"\b(?:void\*|u?int\d+_t|float|double)\s+([^;]*);", body) for n in line.split(",")]
    assert names == [f[0] for f in struct._fields_]


def _frequencies(d, base, scaling, factor, original, low, high):
    if scaling == binding.ROTARY_BASE:
        base = base * factor ** (d / (d - 2))
    out = []
    for i in range(d // 2):
        f, keep = base ** (-2 * i / d), 1.0
        if scaling == binding.ROTARY_LINEAR:
            keep = 0.0
        elif scaling == binding.ROTARY_BANDS:
            keep = (original * f / (2 * math.pi) - low) / (high - low)
        elif scaling == binding.ROTARY_RAMP:
            pair = lambda t: d * math.log(original / (2 * math.pi * t)) / (2 * math.log(base))
            a, b = max(0, math.floor(pair(high))), min(d - 1, math.ceil(pair(low)))
            keep = 1 - (i - a) / max(b - a, 0.001)
        keep = min(max(keep, 0.0), 1.0)
        out.append(f if scaling in (binding.ROTARY_UNSCALED, binding.ROTARY_BASE) else keep * f + (1 - keep) * f / factor)
    return out


@pytest.mark.parametrize("scaling", range(5))
@pytest.mark.parametrize("d,base", [(128, 1.0e4), (16, 5.0e5), (96, 1.0e6)])
def test_rotary_plan_turns(scaling, d, base):
    """turns[i] = f_i / 2 pi rounded to 2^-64 (half of that over f_i / 2 pi is pi 2^-64 / f_i), to the 2^-52 of the 64-bit formula here
    (a few operations, a power among them: 2^-44 is beyond them)."""
    low, high = (1.0, 32.0) if scaling == binding.ROTARY_RAMP else (1.0, 4.0)
    r = binding.rotary_plan(d, base, binding.ROTARY_INTERLEAVED, scaling, 8.0, 8192, low, high)
    for got, f in zip(r.turns, _frequencies(d, base, scaling, 8.0, 8192, low, high)):
        assert abs(got / 2.0 ** 64 / (f / (2 * math.pi)) - 1) < 2.0 ** -44 + math.pi * 2.0 ** -64 / f
    assert not any(r.turns[d // 2:]) and (r.rotary_dim, r.layout) == (d, binding.ROTARY_INTERLEAVED)
    assert abs(r.gain - (0.1 * math.log(8.0) + 1 if scaling == binding.ROTARY_RAMP else 1.0)) < 1e-7
    assert binding.rotary_plan(d, base, gain=0.5).gain == 0.5


@pytest.mark.parametrize("change", [dict(rotary_dim=0), dict(rotary_dim=24), dict(rotary_dim=144), dict(base=1.0), dict(base=math.nan), dict(base=math.inf),
                                    dict(layout=2), dict(scaling=5), dict(scaling=-1), dict(scaling=1, factor=0.5), dict(scaling=1, factor=math.inf),
                                    dict(scaling=3, factor=2.0), dict(scaling=3, factor=2.0, original_tokens=10, low=4.0, high=4.0),
                                    dict(scaling=4, factor=2.0, original_tokens=10, low=0.0, high=4.0), dict(gain=math.nan)])
def test_rotary_plan_refuses(change):
    with pytest.raises(binding.SpeCacheError) as e:
        binding.rotary_plan(**change)
    assert e.value.code == binding.EINVAL and str(e.value).strip()[-1] != ":"


def _rotate(plan=None, dtype=0, batch=1, tokens=2, n_q=2, q=View(A, 512, 256, 128), q_out=View(2 * A, 512, 256, 128), n_kv=1, k=None, k_out=None,
            v=None, v_out=None, positions=None, first=0):
    ref = lambda x: None if x is None else C.byref(x)
    plan = binding.rotary_plan() if plan is None else plan
    return binding.lib().specache_rotate(ref(plan), dtype, batch, tokens, n_q, ref(q), ref(q_out), n_kv, ref(k), ref(k_out), ref(v), ref(v_out),
                                         positions, first, None)


def test_rotate_refuses():
    good = View(A, 512, 256, 128)
    for change in (dict(plan=Rotary()), dict(dtype=2), dict(batch=-1), dict(tokens=-1), dict(n_q=-1), dict(n_kv=-1), dict(q=None), dict(q_out=None),
                   dict(q=View(A + 8, 512, 256, 128)), dict(q=View(A, 512, 256, 132)), dict(q=View(A, 512, -256, 128)), dict(q=View(None, 512, 256, 128)),
                   dict(k=good), dict(v_out=good), dict(q_out=View(A, 512, 128, 256)), dict(q_out=View(2 * A, 512, 256, 0)),
                   dict(first=2 ** 31 - 2), dict(n_q=1 << 21), dict(tokens=(1 << 30) + 1), dict(batch=1 << 24)):
        assert _rotate(**change) == binding.EINVAL, change
        assert binding.lib().specache_last_error(None)
    for nothing in (dict(batch=0), dict(tokens=0), dict(n_q=0)):
        assert _rotate(**nothing) == binding.OK


def _config(**change):
    c = WindowConfig(2, 4, 2, 128, 3, 10, 0, 0, 0, 0.0)
    for k, v in change.items():
        setattr(c, k, v)
    return c


def _window(cfg, q=View(A, 1536, 384, 128), k=View(2 * A, 2560, 1280, 128), v=View(3 * A, 2560, 1280, 128), out=View(4 * A, 1536, 384, 128), scratch=None, size=0):
    ref = lambda x: None if x is None else C.byref(x)
    return binding.lib().specache_window_attend(ref(cfg), ref(q), ref(k), ref(v), ref(out), None, None, scratch, size, None)


def test_window_scratch_of_very_many_rows():
    """A merge of 2^24 rows would have more threads than a launch counts: such calls have no chunks."""
    size = C.c_int64(-7)
    for heads, chunks in ((16, 9), (32, 0)):
        assert binding.lib().specache_window_scratch(C.byref(_config(batch=1 << 19, n_q_heads=heads, n_kv_heads=1, q_tokens=1, kv_tokens=20000)), C.byref(size)) == binding.OK
        assert size.value == (1 << 19) * heads * chunks * (128 + 2) * 4


def test_window_attend_refuses():
    for change in (dict(batch=-1), dict(q_tokens=-1), dict(kv_tokens=-1), dict(window=-1), dict(sinks=-1), dict(n_kv_heads=0), dict(n_q_heads=3), dict(n_q_heads=130),
                   dict(head_dim=64), dict(dtype=2), dict(sm_scale=math.nan), dict(sm_scale=math.inf), dict(kv_tokens=(1 << 28) + 1), dict(q_tokens=1 << 28)):
        assert _window(_config(**change)) == binding.EINVAL, change
        size = C.c_int64(-7)
        assert binding.lib().specache_window_scratch(C.byref(_config(**change)), C.byref(size)) == binding.EINVAL and size.value == -7
    for views in (dict(q=None), dict(k=None), dict(v=None), dict(out=None), dict(k=View(2 * A + 2, 2560, 1280, 128)), dict(out=View(4 * A, 1536, 0, 128)),
                  dict(v=View(3 * A, 2560, 1280, 4)), dict(k=View(2 * A, 0, 0, (1 << 24) + 8))):
        assert _window(_config(), **views) == binding.EINVAL, views
    assert _window(None) == binding.EINVAL
    assert _window(_config(batch=0), q=None) == _window(_config(q_tokens=0), k=None) == binding.OK
    # a step over a long cache needs scratch memory, a prompt none
    long = _config(q_tokens=1, kv_tokens=100000)
    size = C.c_int64()
    assert binding.lib().specache_window_scratch(C.byref(long), C.byref(size)) == binding.OK and size.value > 0
    wide = dict(q=View(A, 512, 128, 128), out=View(4 * A, 512, 128, 128), k=View(2 * A, 1 << 30, 1 << 29, 128), v=View(3 * A, 1 << 30, 1 << 29, 128))
    assert _window(long, **wide) == _window(long, scratch=A + 8, size=size.value, **wide) == binding.EINVAL
    assert _window(long, scratch=A, size=size.value - 1, **wide) == binding.ECAPACITY
    assert binding.window_scratch(1, 32, 32, 16384, 16384) == 0


def _sample(cfg, logits=A, u=A, temperature=None, top_k=None, top_p=None, min_p=None, tokens=A):
    return binding.lib().specache_sample(None if cfg is None else C.byref(cfg), logits, u, temperature, top_k, top_p, min_p, tokens, None, 0, None)


def test_sample_refuses():
    for cfg in (None, SampleConfig(-1, 10, 0, 10), SampleConfig(1, 0, 0, 10), SampleConfig(1, (1 << 20) + 1, 0, 1 << 21), SampleConfig(1, 10, 3, 10), SampleConfig(1, 10, 0, -1)):
        assert _sample(cfg) == binding.EINVAL
        if cfg is not None:
            assert binding.lib().specache_sample_scratch(C.byref(cfg), C.byref(C.c_int64())) == binding.EINVAL
    good = SampleConfig(1, 10, 2, 10)
    for change in (dict(logits=None), dict(logits=A + 2), dict(u=None), dict(u=A + 1), dict(tokens=None), dict(tokens=A + 2), dict(top_k=A + 1), dict(min_p=A + 2)):
        assert _sample(good, **change) == binding.EINVAL, change
    assert _sample(SampleConfig(0, 10, 0, 10), logits=None, u=None, tokens=None) == binding.OK


def test_bindings_refuse_tensors_that_are_not_on_the_device(monkeypatch):
    import torch
    binding._with_torch()
    monkeypatch.setattr(binding, "_here", lambda: 0)
    x = torch.zeros((1, 2, 3, 128), dtype=torch.float16)
    for call in (lambda: binding.rotate(binding.rotary_plan(), x, x), lambda: binding.window_attend(x, x, x, x),
                 lambda: binding.sample(torch.zeros(2, 5), torch.zeros(2), torch.zeros(2, dtype=torch.int32))):
        with pytest.raises(binding.SpeCacheError) as e:
            call()
        assert e.value.code == binding.EINVAL
