"""specache_sample with min_p where more tokens are kept than are listed at once: short rows, whose one pass over the logits is over soon,
so that every wave of a row has to have decided on its way before a faster one goes on."""
import numpy as np
import pytest
import torch

from tests.test_gpu_sample import _check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("V", [2049, 2100, 4099])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_min_p_keeps_more_than_a_list(V, dtype):
    R = 64
    gen = torch.Generator(device="cuda")
    gen.manual_seed(V)
    x = (2.0 * torch.rand((R, V), generator=gen, device="cuda")).to(dtype)     # weights from e^-2 to 1, all above min_p
    u = np.random.default_rng(V).random(R, dtype=np.float32).tolist()
    _check(x, u, m=[0.01] * R)
    _check(x, u, m=[0.01] * R, p=[0.97] * R)
