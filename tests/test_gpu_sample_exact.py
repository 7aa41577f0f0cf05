"""specache_sample against the definition in 64 bits, draw by draw: thousands of random numbers over every row of logits.

The weights of the reference are binary64 exponentials, their running sums 80-bit ones.  The choice has to be the reference's; where u or top_p
lies within NEAR, the library's accuracy (relative to the row's sum), of a border between two tokens, that for either side counts: of a row of 2^17 tokens
some 2^17 * 2^-40 of all draws."""
import numpy as np
import pytest
import torch

from paper_2503_16163_amd import binding

pytestmark = pytest.mark.gpu
NEAR = 2.0 ** -41


class Row:
    """One row's tokens in their order, and the running sums of their weights at a temperature."""

    def __init__(self, x, t):
        x = x.astype(np.float64)
        order = np.argsort(-x, kind="stable")
        self.order = order = order[x[order] > -np.inf]
        self.weights = np.exp((x[order] - x[order[0]]) / np.float64(np.float32(t)))
        self.sums = np.cumsum(self.weights.astype(np.longdouble))

    def choices(self, u, k=0, p=1.0, m=0.0):
        """Tokens for an array of random numbers."""
        n = min(k, len(self.sums)) if k > 0 else len(self.sums)
        if p < 1:
            n = min(n, 1 + int(np.searchsorted(self.sums[:n], np.longdouble(p) * self.sums[n - 1], side="left")))
        if m > 0:
            n = min(n, max(1, int((self.weights >= m).sum())))
        at = np.searchsorted(self.sums[:n], u.astype(np.longdouble) * self.sums[n - 1], side="right")
        return self.order[np.minimum(at, n - 1)]


def _draw(x, u, t, k=0, p=1.0, m=0.0):
    """x: one row of logits; u: host array of random numbers."""
    R = len(u)
    all_rows = lambda a, kind: torch.full((R,), a, dtype=kind, device="cuda")
    tokens = torch.full((R,), -5, dtype=torch.int32, device="cuda")
    binding.sample(x.view(1, -1).expand(R, -1), torch.from_numpy(u).cuda(), tokens, all_rows(t, torch.float32), all_rows(k, torch.int32),
                   all_rows(p, torch.float32), all_rows(m, torch.float32))
    return tokens.cpu().numpy()


def _check(x, t, k, p, m, u):
    got, row = _draw(x, u, t, k, p, m), Row(x.float().cpu().numpy(), t)
    p, m, wide = float(np.float32(p)), float(np.float32(m)), u.astype(np.float64)
    right = np.zeros(len(u), dtype=bool)
    for a in (0, -1, 1):
        for b in (0, -1, 1) if p < 1 else (0,):
            right |= got == row.choices(wide * (1 + a * NEAR), k, p * (1 + b * NEAR) if p < 1 else p, m)
    wrong = np.nonzero(~right)[0]
    assert len(wrong) == 0, (len(wrong), len(u), [(float(u[i]), int(got[i]), int(row.choices(wide[i:i + 1], k, p, m)[0])) for i in wrong[:3]])


def _logits(seed, V, dtype, sigma=2.5):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    x = sigma * torch.randn((V,), generator=gen, device="cuda")
    x[torch.randint(0, V, (12,), generator=gen, device="cuda")] = 8 + 6 * torch.rand((12,), generator=gen, device="cuda")
    return x.to(dtype)


DRAWS = 8192


@pytest.mark.parametrize("t", [0.7, 1.0, 1.3, 2.0])
@pytest.mark.parametrize("V,dtype", [(32000, torch.float16), (128256, torch.bfloat16), (128256, torch.float32), (1 << 20, torch.bfloat16), (1 << 20, torch.float32)])
def test_every_draw_is_the_definitions(V, dtype, t):
    """10^6 draws in all: without limits, with top_p, with min_p, with top_k of both kinds."""
    rng = np.random.default_rng(V)
    x = _logits(V + 1, V, dtype)
    for k, p, m in ((0, 1.0, 0.0), (0, 0.95, 0.0), (0, 0.5, 0.0), (0, 0.97, 1e-5), (0, 1.0, 1e-4), (1000, 0.9, 0.0), (20000, 1.0, 0.0), (20000, 0.99, 1e-7)):
        _check(x, t, k, p, m, rng.random(DRAWS, dtype=np.float32))


def test_logits_and_temperatures_over_the_whole_range():
    """Differences that binary32 does not hold, temperatures from its least to infinity: the weights are the definition's."""
    rng = np.random.default_rng(3)
    big = 3.0e38
    x = torch.tensor([big, -big, 0.0, 1.0e38, 2.0e38, -1.0, big, 1.0e-30, -1.0e38] * 700, device="cuda")
    for t in (1.0e-45, 1.0, 1.0e30, 1.0e37, 1.0e38, 3.0e38, np.inf):
        for k, p, m in ((0, 1.0, 0.0), (5, 1.0, 0.0), (2000, 0.9, 0.0), (4000, 0.7, 0.0), (0, 0.6, 0.2), (0, 1.0, 0.3)):
            _check(x, t, k, p, m, rng.random(256, dtype=np.float32))
    x = torch.arange(3000, device="cuda", dtype=torch.float32) * 2.0 ** -20 + 1.0
    for t in (2.0 ** -22, 2.0 ** -12, 1.0e-3):
        for k, p, m in ((0, 1.0, 0.0), (100, 0.9, 0.0), (0, 0.97, 0.0), (2500, 0.99, 0.0)):
            _check(x, t, k, p, m, rng.random(256, dtype=np.float32))


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16, torch.float32])
@pytest.mark.parametrize("V", [3, 2000, 40000])
def test_rows_of_the_lowest_number(V, dtype):
    """Masked by the type's lowest number instead of -infinity: it is a logit like others, beside larger ones of no weight, alone of equal weight."""
    rng = np.random.default_rng(V)
    u = rng.random(64, dtype=np.float32)
    x = torch.full((V,), torch.finfo(dtype).min, dtype=dtype, device="cuda")
    for k, p, m in ((0, 1.0, 0.0), (2, 1.0, 0.0), (300, 0.5, 0.0), (0, 0.7, 0.5), (1900, 0.9, 1.0)):
        _check(x, 1.0, k, p, m, u)
    x[V // 2] = -5.0
    x[V // 3] = -6.0
    for k, p, m in ((0, 1.0, 0.0), (1, 1.0, 0.0), (300, 0.5, 0.0), (0, 0.9, 0.1), (1900, 0.99, 0.0)):
        _check(x, 1.0, k, p, m, u)
