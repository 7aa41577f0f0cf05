"""specache_paged_attend where a prefix is worked on for all sequences together: sizes at which the call chooses to (each test asks for that first), against 64 bits.

Whether it does shows in the scratch memory that it asks for: the prefix's partial results are in it.  Tolerances are those of tests/paged.py's reference."""
import math

import pytest
import torch

from paper_2503_16163_amd import binding
from tests.paged import attend, compare, generator, ints, pool, reference, scratch_of, table_of

pytestmark = pytest.mark.gpu
SCALE = 128 ** -0.5
KINDS = {   # B, Hq, Hkv, queries, longest, page, shared
    "steps": (8, 32, 8, 1, 6300, 32, 6144), "steps_odd": (5, 8, 8, 3, 17001, 16, 16390), "mixed": (32, 16, 8, 3, 2311, 64, 2100), "mixed_many": (33, 32, 8, 2, 4444, 16, 4100),
    "mixed_two_to_a_unit": (32, 32, 8, 8, 16500, 256, 16384), "tiles_4": (16, 8, 8, 34, 1200, 64, 1030), "tiles_4_long": (12, 8, 8, 40, 2300, 32, 2100),
    "tiles_8": (8, 8, 4, 130, 4400, 128, 4100),
}
FEW = ["steps", "mixed", "tiles_4", "tiles_8"]


def _make(kind, seed, dtype, order="heads"):
    B, Hq, Hkv, n, most, page, shared = KINDS[kind]
    gen = generator(seed)
    table, pages = table_of(gen, [most] * B, page, -(-most // page), shared // page)
    k, v = pool(gen, pages, Hkv, page, dtype, order)
    q = torch.randn((B, Hq, n, 128), generator=gen, device="cuda").to(dtype)
    cache = binding.Pages(k, v, table)
    assert binding.paged_scratch(cache, B, Hq, n, most, shared) != binding.paged_scratch(cache, B, Hq, n, most, 0), "this size does not share"
    return q, k, v, table, cache


def _lengths(kind):
    """Of every sequence: from the shared positions and its own queries on to the longest."""
    B, _, _, n, most, _, shared = KINDS[kind]
    return [most - (most - shared - n) * b // B for b in range(B)]


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("kind", KINDS)
def test_a_prefix_of_all(kind, dtype):
    B, _, _, n, most, _, shared = KINDS[kind]
    q, k, v, table, cache = _make(kind, 1, dtype, "places" if n % 2 else "heads")
    N_of = _lengths(kind)
    exact, tol = reference(q, k, v, table, [n] * B, N_of, SCALE)
    compare(attend(cache, q, most, shared, None, N_of), exact, tol, [n] * B)
    compare(attend(cache, q, most, 0, None, N_of), exact, tol, [n] * B)


@pytest.mark.parametrize("kind", FEW)
def test_sequences_that_end_inside_it_or_have_nothing(kind):
    B, _, _, n, most, page, shared = KINDS[kind]
    q, k, v, table, cache = _make(kind, 2, torch.bfloat16)
    N_of, n_of = _lengths(kind), [n] * B
    N_of[1], N_of[2], N_of[3], n_of[4] = 0, 1, shared // 2 + 3, 0
    for b in range(B):
        q[b, :, n_of[b]:] = math.nan
    exact, tol = reference(q, k, v, table, n_of, N_of, SCALE)
    compare(attend(cache, q, most, shared, n_of, N_of), exact, tol, n_of)


@pytest.mark.parametrize("kind", FEW)
def test_missing_pages_and_values_that_are_not_finite(kind):
    B, _, Hkv, n, most, page, shared = KINDS[kind]
    q, k, v, table, cache = _make(kind, 3, torch.bfloat16)
    table[:, 1], table[:, 5], table[2, -1] = -1, 1 << 20, -1      # two of what is shared, one sequence's last
    v[table[0, 2].item(), 0, 3, 7] = math.inf                     # of what is shared: all rows of one head see it
    v[table[1, -1].item(), Hkv - 1, 1, 9] = math.nan              # of one sequence's own
    N_of = _lengths(kind)
    exact, tol = reference(q, k, v, table, [n] * B, N_of, SCALE)
    compare(attend(cache, q, most, shared, None, N_of), exact, tol, [n] * B)
    table.fill_(-1)
    assert bool((attend(cache, q, most, shared, None, N_of) == 0).all())


@pytest.mark.parametrize("kind", FEW)
def test_captured_and_the_same_every_time(kind):
    """Replays while lengths change; scratch memory holds what an earlier call left."""
    B, Hq, _, n, most, _, shared = KINDS[kind]
    q, k, v, table, cache = _make(kind, 4, torch.float16)
    lengths, out = ints(_lengths(kind)), torch.full_like(q, 7.0)
    scratch = scratch_of(binding.paged_scratch(cache, B, Hq, n, most, shared))
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        binding.paged_attend(cache, q, out, most, shared, kv_lengths=lengths, scratch=scratch, stream=torch.cuda.current_stream())
    for i in range(3):
        lengths.sub_(i)
        q.copy_(q.flip(2) if i else q)
        want = attend(cache, q, most, shared, None, lengths.tolist())
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)


@pytest.mark.parametrize("kind", FEW)
def test_nothing_but_what_is_shared(kind):
    """The longest sequence ends where the shared pages do (their queries then see less of them than all), and the others before."""
    B, Hq, Hkv, n, most, page, shared = KINDS[kind]
    q, k, v, table, cache = _make(kind, 5, torch.bfloat16)
    whole = shared // page * page
    N_of = [whole - b for b in range(B)]
    assert binding.paged_scratch(cache, B, Hq, n, whole, shared) != binding.paged_scratch(cache, B, Hq, n, whole, 0), "this size does not share"
    exact, tol = reference(q, k, v, table, [n] * B, N_of, SCALE)
    compare(attend(cache, q, whole, shared, None, N_of), exact, tol, [n] * B)
