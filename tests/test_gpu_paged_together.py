"""The calls on a paged cache as a server makes them: a system prompt is appended once and shared, each sequence's question follows as a part of a prompt, then steps
of several sequences append, attend behind the shared prefix, choose blocks and attend to those, and choose tokens; at last a step in a graph."""
import math

import pytest
import torch

from paper_2503_16163_amd import binding
from tests.paged import compare, generator, ints, reference, scratch_of
from tests.test_gpu_blocks import _seen, lists
from tests.test_gpu_sample import _choices

pytestmark = pytest.mark.gpu
HQ, HKV, PAGE, WIDTH, VOCAB = 8, 2, 32, 24, 3001
SCALE = 1 / math.sqrt(128)


def _project(gen, B, n, kind):
    x = torch.randn((B, n, HQ + 2 * HKV, 128), generator=gen, device="cuda").to(kind).transpose(1, 2)
    return x[:, :HQ], x[:, HQ:HQ + HKV], x[:, HQ + HKV:]


@pytest.mark.parametrize("kind,scaling", [(torch.float16, binding.ROTARY_UNSCALED), (torch.bfloat16, binding.ROTARY_BANDS)])
def test_shared_prompt_questions_and_steps(kind, scaling):
    gen = generator(5)
    B, S, asked, steps = 3, 421, [60, 1, 33], 40
    plan = binding.rotary_plan(128, 5.0e5, scaling=scaling, factor=8.0, original_tokens=8192, low=1.0, high=4.0)
    n_pages, full = 100, S // PAGE
    k, v = (torch.full((n_pages, HKV, PAGE, 128), math.nan, device="cuda", dtype=kind) for _ in range(2))
    bounds = torch.full((n_pages, HKV, 2, 128), math.nan, device="cuda", dtype=kind)
    order = torch.randperm(n_pages, generator=gen, device="cuda").to(torch.int32)
    table = torch.full((B, WIDTH), -1, dtype=torch.int32, device="cuda")
    table[:, :full] = order[:full]
    for b in range(B):
        table[b, full:] = order[full + b * (WIDTH - full):full + (b + 1) * (WIDTH - full)]
    cache = binding.Pages(k, v, table, bounds)

    # the system prompt, to the first sequence; the others take its full pages as they are and a copy of the last one
    one = binding.Pages(k, v, table[:1], bounds)
    q, k_new, v_new = _project(gen, 1, S, kind)
    turned = torch.empty(q.shape, device="cuda", dtype=kind)
    binding.paged_append(one, plan, k_new, v_new, q, turned)
    out = torch.full(q.shape, 7.0, device="cuda", dtype=kind)
    binding.paged_attend(one, turned, out, S, scratch=scratch_of(binding.paged_scratch(one, 1, HQ, S, S)))
    exact, tol = reference(turned, k, v, table, [S], [S], SCALE)
    compare(out, exact, tol, [S])
    for pages in (k, v, bounds):
        for b in range(1, B):
            pages[table[b, full].long()] = pages[table[0, full].long()]

    # the questions
    cached = [S + n for n in asked]
    q, k_new, v_new = _project(gen, B, max(asked), kind)
    turned = torch.full(q.shape, 7.0, device="cuda", dtype=kind)
    binding.paged_append(cache, plan, k_new, v_new, q, turned, ints([S] * B), ints(asked))
    out = torch.full(q.shape, 7.0, device="cuda", dtype=kind)
    most = S + max(asked)
    binding.paged_attend(cache, turned, out, most, S, ints(asked), ints(cached), scratch=scratch_of(binding.paged_scratch(cache, B, HQ, max(asked), most, S)))
    exact, tol = reference(turned, k, v, table, asked, cached, SCALE)
    compare(out, exact, tol, asked)

    # steps
    most = max(cached) + steps
    scratch = scratch_of(max(binding.paged_scratch(cache, B, HQ, 1, most, S), binding.block_scratch(cache, B, HQ, 1, most, 4, 1, 2)))
    weight = torch.randn((VOCAB, HQ * 128), generator=gen, device="cuda") * 0.1
    blocks = torch.empty((B, HKV, 1, 7), dtype=torch.int32, device="cuda")
    for t in range(steps):
        q, k_new, v_new = _project(gen, B, 1, kind)
        turned = torch.empty(q.shape, device="cuda", dtype=kind)
        binding.paged_append(cache, plan, k_new, v_new, q, turned, ints(cached))
        cached = [N + 1 for N in cached]
        N = ints(cached)
        out, sparse = (torch.full(q.shape, 7.0, device="cuda", dtype=kind) for _ in range(2))
        binding.paged_attend(cache, turned, out, most, S, kv_lengths=N, scratch=scratch)
        binding.block_select(cache, turned, blocks, most, 4, 1, 2, kv_lengths=N, scratch=scratch)
        binding.block_attend(cache, turned, sparse, blocks, most, kv_lengths=N, scratch=scratch)
        if t % 9 == 0 or t == steps - 1:
            exact, tol = reference(turned, k, v, table, [1] * B, cached, SCALE)
            compare(out, exact, tol, [1] * B)
            # a page's bounds are those of the keys that it holds
            for b, n in enumerate(cached):
                for i in range(-(-n // PAGE)):
                    held = k[table[b, i].long(), :, :min(PAGE, n - i * PAGE)]
                    assert torch.equal(bounds[table[b, i].long(), :, 0], held.amin(dim=1)) and torch.equal(bounds[table[b, i].long(), :, 1], held.amax(dim=1))
            assert torch.equal(blocks, lists(turned, bounds, table, [1] * B, cached, PAGE, 4, 1, 2))
            exact, tol = reference(turned, k, v, table, [1] * B, cached, SCALE, _seen(blocks, PAGE, cached))
            compare(sparse, exact, tol, [1] * B)
            logits = out.float().transpose(1, 2).reshape(B, -1) @ weight.t()
            u, tokens = torch.rand(B, generator=gen, device="cuda"), torch.zeros(B, dtype=torch.int32, device="cuda")
            binding.sample(logits, u, tokens, top_p=torch.full((B,), 0.9, device="cuda"))
            for r, token in enumerate(tokens.tolist()):
                assert token in _choices(logits[r].double().cpu().numpy(), u[r].item(), 1.0, 0, 0.9, 0.0)


def test_a_step_in_a_graph():
    """Append, attention behind the shared prefix, choice of blocks and attention to them, captured once and replayed while the sequences grow."""
    gen = generator(6)
    B, S, most, kind = 4, 256, 700, torch.bfloat16
    plan, n_pages = binding.rotary_plan(), 100
    table = torch.randperm(n_pages, generator=gen, device="cuda")[:B * WIDTH].view(B, WIDTH).to(torch.int32)
    table[:, :S // PAGE] = table[0, :S // PAGE]
    start_k, start_v = (torch.randn((n_pages, HKV, PAGE, 128), generator=gen, device="cuda").to(kind) for _ in range(2))
    start_bounds = torch.stack([start_k.amin(dim=2), start_k.amax(dim=2)], dim=2)
    sets = []
    for i in range(2):                      # eager, captured
        k, v, bounds = start_k.clone(), start_v.clone(), start_bounds.clone()
        cache = binding.Pages(k, v, table, bounds)
        sets.append(dict(k=k, v=v, bounds=bounds, cache=cache, q=torch.zeros((B, HQ, 1, 128), device="cuda", dtype=kind), out=torch.zeros((B, HQ, 1, 128), device="cuda", dtype=kind),
                         sparse=torch.zeros((B, HQ, 1, 128), device="cuda", dtype=kind), blocks=torch.zeros((B, HKV, 1, 7), dtype=torch.int32, device="cuda"),
                         scratch=scratch_of(max(binding.paged_scratch(cache, B, HQ, 1, most, S), binding.block_scratch(cache, B, HQ, 1, most, 4, 1, 2)))))
    x = torch.randn((B, 1, HQ + 2 * HKV, 128), generator=gen, device="cuda").to(kind).transpose(1, 2)
    held, seen = torch.tensor([300, 280, 257, 400], dtype=torch.int32, device="cuda"), torch.zeros(B, dtype=torch.int32, device="cuda")

    def step(s):
        torch.add(held, 1, out=seen)
        binding.paged_append(s["cache"], plan, x[:, HQ:HQ + HKV], x[:, HQ + HKV:], x[:, :HQ], s["q"], held)
        binding.paged_attend(s["cache"], s["q"], s["out"], most, S, kv_lengths=seen, scratch=s["scratch"])
        binding.block_select(s["cache"], s["q"], s["blocks"], most, 4, 1, 2, kv_lengths=seen, scratch=s["scratch"])
        binding.block_attend(s["cache"], s["q"], s["sparse"], s["blocks"], most, kv_lengths=seen, scratch=s["scratch"])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(sets[1])
    for turn in range(40):
        x.copy_(torch.randn_like(x))
        step(sets[0])
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for name in ("q", "out", "sparse", "blocks", "k", "v", "bounds"):
            assert torch.equal(sets[0][name], sets[1][name]), (turn, name)
        held.add_(1)
