"""The calls without a context are enqueued on torch's current stream where none is given.  On the CPU: the library is replaced by a recorder, and tensors
of the host stand for the device's."""
import pytest
import torch

from paper_2503_16163_amd import binding


class _Recorder:
    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        def call(*args):
            self.calls.append((name, args))
            return binding.OK
        return call


class _Stream:
    cuda_stream = 0x5EED


@pytest.fixture
def calls(monkeypatch):
    recorder = _Recorder()
    binding._with_torch()
    monkeypatch.setattr(binding, "_here", lambda: -1)          # (get_device() of a host tensor)
    monkeypatch.setattr(binding, "lib", lambda: recorder)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: _Stream)
    return recorder.calls


def _all(stream):
    x = torch.zeros((1, 2, 3, 128), dtype=torch.float16)
    binding.rotate(binding.Rotary(), x, x, **stream)
    binding.window_attend(x, x, x, x, **stream)
    binding.sample(torch.zeros(2, 5), torch.zeros(2), torch.zeros(2, dtype=torch.int32), **stream)


def test_the_current_stream_is_the_default(calls):
    _all({})
    _all({"stream": None})
    assert [name for name, _ in calls] == ["specache_rotate", "specache_window_attend", "specache_sample"] * 2
    assert all(args[-1] == 0x5EED for _, args in calls)


@pytest.mark.parametrize("given,want", [(0, 0), (77, 77), (_Stream, 0x5EED)])
def test_a_given_stream_is_taken(calls, given, want):
    _all({"stream": given})
    assert all(args[-1] == want for _, args in calls)


@pytest.mark.gpu
def test_under_a_stream_and_captured_without_naming_it():
    gen = torch.Generator(device="cuda")
    gen.manual_seed(3)
    make = lambda *s: torch.randn(s, generator=gen, device="cuda", dtype=torch.float16)
    plan, x, k, v = binding.rotary_plan(), make(2, 8, 40, 128), make(2, 2, 40, 128), make(2, 2, 40, 128)
    logits, u = make(4, 3000).float(), torch.tensor([0.1, 0.4, 0.6, 0.9], device="cuda")
    y, out, tokens = torch.empty_like(x), torch.empty_like(x), torch.zeros(4, dtype=torch.int32, device="cuda")
    need = binding.window_scratch(2, 8, 2, 40, 40)
    scratch = torch.empty(need, dtype=torch.uint8, device="cuda") if need else None
    top_p = torch.full_like(u, 0.9)

    def step():
        binding.rotate(plan, x, y, first_position=5)
        binding.window_attend(y, k, v, out, scratch=scratch)
        binding.sample(logits, u, tokens, top_p=top_p)
    step()
    torch.cuda.synchronize()
    want = (y.clone(), out.clone(), tokens.clone())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    stream = torch.cuda.Stream()
    for run in (graph.replay, step):
        for t in (y, out, tokens):
            t.zero_()
        stream.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(stream):
            run()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, (y, out, tokens)))
