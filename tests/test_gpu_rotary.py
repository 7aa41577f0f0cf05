"""specache_rotate against the formulas in 64 bits.

Tolerance: the result is rounded once to its type (half a step of |y|, in binary16 at least half the smallest number), before that
two products and a sum in binary32 of operands whose cosine and sine are off by the angle's 2^-25 turns and the hardware functions'
error, taken as 2^-19 together: 2^-18 of gain * hypot(x1, x2)."""
import math

import pytest
import torch

from paper_2503_16163_amd import binding
from tests.test_operators import _frequencies

pytestmark = pytest.mark.gpu


def _bound(y, x, gain, dtype, d, layout):
    first, second = _pairs(d, layout)
    h = torch.zeros_like(y)
    r = torch.hypot(x[..., first], x[..., second]) * gain
    h[..., first] = r
    h[..., second] = r
    least = 2.0 ** -25 if dtype == torch.float16 else 0.0
    return (torch.finfo(dtype).eps / 2 * (y.abs() + 2.0 ** -18 * h)).clamp(min=least) + 2.0 ** -18 * h


def _pairs(d, layout):
    if layout == binding.ROTARY_HALF:
        return list(range(d // 2)), list(range(d // 2, d))
    return list(range(0, d, 2)), list(range(1, d, 2))


def _expected(x, positions, f, gain, d, layout):
    angle = positions.double()[:, None, :, None] * torch.tensor(f, dtype=torch.float64, device=x.device)
    z = x.double().clone()
    first, second = _pairs(d, layout)
    t = torch.complex(z[..., first], z[..., second]) * torch.polar(torch.full_like(angle, gain), angle)
    z[..., first], z[..., second] = t.real, t.imag
    return z


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("layout", [0, 1])
@pytest.mark.parametrize("B,L,Hq,Hkv,d,scaling", [(1, 1, 1, 1, 128, 0), (1, 2, 32, 8, 128, 3), (3, 5, 5, 5, 64, 1), (2, 33, 8, 1, 96, 4), (1, 1000, 16, 4, 16, 2), (2, 257, 7, 7, 112, 0)])
def test_rotate(B, L, Hq, Hkv, d, scaling, layout, dtype):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(B * 1000 + L)
    low, high = (1.0, 32.0) if scaling == binding.ROTARY_RAMP else (1.0, 4.0)
    plan = binding.rotary_plan(d, 1.0e4, layout, scaling, 8.0, 4096, low, high)
    f = _frequencies(d, 1.0e4, scaling, 8.0, 4096, low, high)
    x = torch.randn((B, L, Hq + 2 * Hkv, 128), generator=gen, device="cuda").to(dtype).transpose(1, 2)
    q, k, v = x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:]
    positions = torch.randint(-1000, 2 ** 20, (B, L), generator=gen, device="cuda", dtype=torch.int32)
    q_out, k_out, v_out = (torch.full(t.shape, math.nan, device="cuda", dtype=dtype) for t in (q, k, v))
    binding.rotate(plan, q, q_out, k, k_out, v, v_out, positions=positions)
    for y, t in ((q_out, q), (k_out, k)):
        e = _expected(t, positions, f, plan.gain, d, layout)
        assert bool(((y.double() - e).abs()[..., :d] <= _bound(e, t.double(), plan.gain, dtype, d, layout)[..., :d]).all())
        assert torch.equal(y[..., d:], t[..., d:])
    assert torch.equal(v_out, v)
    # positions in a row, and in place
    want = torch.empty_like(q_out)
    row = 77 + torch.arange(L, device="cuda", dtype=torch.int32).repeat(B, 1)
    binding.rotate(plan, q, want, positions=row.contiguous())
    binding.rotate(plan, q, q, k, k, first_position=77)
    assert torch.equal(q, want) and torch.equal(x[:, Hq + Hkv:], v_out)


def test_far_positions_and_special_values():
    """Positions at the ends of int32 (the 64-bit formula's own angle is off by 2^31 * 2^-52 there), values that are not finite stay in their pair."""
    plan = binding.rotary_plan()
    f = _frequencies(128, 1.0e4, 0, 1.0, 0, 0, 0)
    x = torch.randn((1, 2, 4, 128), device="cuda", dtype=torch.bfloat16)
    positions = torch.tensor([[2 ** 31 - 1, -2 ** 31, 0, 10 ** 9]], device="cuda", dtype=torch.int32)
    y = torch.empty_like(x)
    binding.rotate(plan, x, y, positions=positions)
    e = _expected(x, positions, f, 1.0, 128, 0)
    assert bool(((y.double() - e).abs() <= _bound(e, x.double(), 1.0, torch.bfloat16, 128, 0)).all())
    assert torch.equal(y[:, :, 2], x[:, :, 2])
    x[0, 0, 0, 5] = math.inf
    x[0, 1, 3, 9] = math.nan
    z = torch.empty_like(x)
    binding.rotate(plan, x, z, positions=positions)
    same = torch.ones((1, 2, 4, 128), dtype=torch.bool, device="cuda")
    for c in (5, 5 + 64):
        same[0, 0, 0, c] = False
    for c in (9, 9 + 64):
        same[0, 1, 3, c] = False
    assert torch.equal(z[same], y[same]) and not bool(torch.isfinite(z[~same]).any())


def test_rows_beyond_32_bit_offsets():
    """Token and head strides that take a row's offset past 2^32 bytes."""
    flat = torch.empty(5 * (1 << 30) // 2 + 4096, device="cuda", dtype=torch.bfloat16)
    far = flat.as_strided((1, 3, 3, 128), (0, 1 << 30, 1 << 28, 1))
    far.copy_(torch.randn((1, 3, 3, 128), device="cuda"))
    near, got = torch.empty((1, 3, 3, 128), device="cuda", dtype=torch.bfloat16), torch.empty((1, 3, 3, 128), device="cuda", dtype=torch.bfloat16)
    plan = binding.rotary_plan()
    binding.rotate(plan, far.contiguous(), near, first_position=3)
    binding.rotate(plan, far, got, first_position=3)
    assert torch.equal(near, got)
    binding.rotate(plan, far, far, first_position=3)
    assert torch.equal(near, far)


def test_more_tokens_than_small_tiles_take():
    """2^26 + 5 tokens that share their input row: the output's rows are those of shorter calls at the same positions."""
    n, plan = (1 << 26) + 5, binding.rotary_plan()
    x = torch.randn((1, 1, 1, 128), device="cuda").to(torch.bfloat16)
    out = torch.zeros((1, 1, n, 128), device="cuda", dtype=torch.bfloat16)
    binding.rotate(plan, x.expand(1, 1, n, 128), out, first_position=11)
    for at in (0, 1 << 20, (1 << 25) + 3, n - 4099):
        part = torch.empty((1, 1, 4099, 128), device="cuda", dtype=torch.bfloat16)
        binding.rotate(plan, x.expand(1, 1, 4099, 128), part, first_position=11 + at)
        assert torch.equal(out[:, :, at:at + 4099], part)


def test_captured_and_on_another_stream():
    plan = binding.rotary_plan(64, layout=binding.ROTARY_INTERLEAVED)
    x = torch.randn((2, 8, 40, 128), device="cuda", dtype=torch.float16)
    positions = torch.arange(80, device="cuda", dtype=torch.int32).view(2, 40)
    y, want = torch.empty_like(x), torch.empty_like(x)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        binding.rotate(plan, x, y, positions=positions, stream=torch.cuda.current_stream())
    for i in range(3):
        x.copy_(torch.randn_like(x))
        positions.add_(1000)
        binding.rotate(plan, x, want, positions=positions)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want)
