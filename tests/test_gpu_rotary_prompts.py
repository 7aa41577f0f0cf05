"""specache_rotate on prompts whose workgroups walk all heads, several rows of a lane in flight and more than once around, and whose outputs are stored past the
caches: every element against the 64-bit formula, in both types and layouts, with odd numbers of heads, and in place."""
import pytest
import torch

from paper_2503_16163_amd import binding
from tests.test_gpu_rotary import _bound, _expected
from tests.test_operators import _frequencies

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("layout", [0, 1])
@pytest.mark.parametrize("B,L,Hq,Hkv,d", [(1, 20000, 32, 8, 128), (1, 20001, 31, 7, 64), (2, 9999, 33, 1, 96), (1, 300, 64, 64, 128)])
def test_prompts(B, L, Hq, Hkv, d, layout, dtype):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(L)
    plan, f = binding.rotary_plan(d, 5.0e5, layout), _frequencies(d, 5.0e5, 0, 1.0, 0, 0, 0)
    x = torch.randn((B, L, Hq + 2 * Hkv, 128), generator=gen, device="cuda").to(dtype).transpose(1, 2)
    q, k, v = x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:]
    positions = torch.randint(0, 2 ** 20, (B, L), generator=gen, device="cuda", dtype=torch.int32)
    q_out, k_out, v_out = (torch.full(t.shape, float("nan"), device="cuda", dtype=dtype) for t in (q, k, v))
    binding.rotate(plan, q, q_out, k, k_out, v, v_out, positions=positions)
    assert torch.equal(v_out, v)
    for y, t in ((q_out, q), (k_out, k)):
        for h in range(0, t.shape[1], 8):
            part, got = t[:, h:h + 8], y[:, h:h + 8]
            e = _expected(part, positions, f, plan.gain, d, layout)
            assert bool(((got.double() - e).abs() <= _bound(e, part.double(), plan.gain, dtype, d, layout))[..., :d].all())
            assert torch.equal(got[..., d:], part[..., d:])
    # in place, all three of the projection's own rows
    binding.rotate(plan, q, q, k, k, v, v, positions=positions)
    assert torch.equal(q, q_out) and torch.equal(k, k_out) and torch.equal(v, v_out)


@pytest.mark.parametrize("L", [37, 20000])
def test_a_tensor_left_out(L):
    """k without v and v without k give what the call with all three gives."""
    plan = binding.rotary_plan()
    q, k, v = (torch.randn((1, h, L, 128), generator=torch.Generator(device="cuda").manual_seed(h), device="cuda", dtype=torch.bfloat16) for h in (8, 3, 3))
    all_out, some = [torch.empty_like(t) for t in (q, k, v)], [torch.empty_like(t) for t in (q, k, v)]
    binding.rotate(plan, q, all_out[0], k, all_out[1], v, all_out[2], first_position=9)
    binding.rotate(plan, q, some[0], k, some[1], first_position=9)
    assert torch.equal(some[0], all_out[0]) and torch.equal(some[1], all_out[1])
    binding.rotate(plan, q, some[0], v=v, v_out=some[2], first_position=9)
    assert torch.equal(some[0], all_out[0]) and torch.equal(some[2], v)
