"""specache_sample with a min_p that no token reaches (above 1, infinite): one token is kept, the first in the row's order."""
import math

import pytest
import torch

from tests.test_gpu_sample import _call

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("value", [2.0, 0.0, -7.0, math.inf])
@pytest.mark.parametrize("V", [5, 4000])
def test_only_the_first_of_equal_tokens(V, value):
    x = torch.full((4, V), -100.0, device="cuda")
    x[:, 1] = value
    x[:, 3:] = value
    u = [0.0, 0.4, 0.8, 0.99]
    for m in (1.0000001, 1.5, 100.0, math.inf):
        assert _call(x, u, m=[m] * 4) == [1, 1, 1, 1]
        assert _call(x, u, k=[3] * 4, p=[0.9] * 4, m=[m] * 4) == [1, 1, 1, 1]
    # at 1 every one of them is kept
    assert _call(x, u, m=[1.0] * 4) == _call(x, u) != [1, 1, 1, 1]
