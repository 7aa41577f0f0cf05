"""specache_sample over vocabularies up to the largest, where a row has more vectors than their table holds (fp32 beyond 131072 tokens, 16 bits beyond 262144) and the
units of a weight are fewest: every draw is the definition's."""
import numpy as np
import pytest
import torch

from tests.test_gpu_sample import _call
from tests.test_gpu_sample_exact import _check, _draw, _logits

pytestmark = pytest.mark.gpu
VOCABULARIES = [131071, 131073, 151936, 262143, 262147, (1 << 20) - 1, 1 << 20]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", VOCABULARIES)
def test_limits(V, dtype):
    rng = np.random.default_rng(V)
    x = _logits(V, V, dtype)
    for t in (1.0, 3.0, 20.0):
        for k in (1, 255, 256, 257, 511, 512, 513, 1535, 1536, 1537, 5000, V - 1, V, V + 1):
            _check(x, t, k, 1.0, 0.0, rng.random(64, dtype=np.float32))
        for k, p, m in ((0, 1.0, 0.0), (0, 0.9, 0.0), (0, 0.999, 0.0), (0, 1.0, 1e-3), (0, 0.99, 1e-6), (512, 0.9, 1e-3), (1537, 0.9, 0.0), (70000, 0.95, 1e-7)):
            _check(x, t, k, p, m, rng.random(256, dtype=np.float32))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [131073, 262147, 1 << 20])
def test_rows_of_equal_logits(V, dtype):
    """Whole numbers of equal weights: no rounding decides, whatever the limits."""
    x = torch.full((5, V), -3.25, dtype=dtype, device="cuda")
    u = [0.0, 0.25, 0.5, 0.7, 1 - 2.0 ** -24]
    number = lambda n: [int(n * float(np.float32(a))) for a in u]
    assert _call(x, u) == number(V)
    for k in (256, 512, 1536, 1537, 100000):
        assert _call(x, u, k=[k] * 5) == number(k)
    assert _call(x, u, p=[0.5] * 5) == number((V + 1) // 2)
    assert _call(x, u, m=[0.5] * 5) == number(V) and _call(x, u, k=[100000] * 5, p=[0.5] * 5, m=[1.0] * 5) == number(50000)


@pytest.mark.parametrize("V", [151936, 1 << 20])
def test_mostly_masked(V):
    """One token in a thousand allowed, and one alone."""
    rng = np.random.default_rng(V)
    x = _logits(V + 5, V, torch.float32)
    hidden = torch.rand((V,), generator=torch.Generator(device="cuda").manual_seed(V), device="cuda") > 0.001
    x[hidden] = -np.inf
    for k, p, m in ((0, 1.0, 0.0), (0, 0.9, 0.0), (300, 1.0, 0.0), (5000, 0.99, 1e-3)):
        _check(x, 1.3, k, p, m, rng.random(256, dtype=np.float32))
    x[:] = -np.inf
    x[V - 1] = -1.0e38
    assert (_draw(x, np.array([0.0, 0.5, 1 - 2.0 ** -24], dtype=np.float32), 1.0) == V - 1).all()
