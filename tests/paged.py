"""Paged caches for the tests, and what attention over them is in 64 bits."""
import math

import torch

from paper_2503_16163_amd import binding


def generator(seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return gen


def pool(gen, pages, Hkv, page, dtype, order="heads", fill=True):
    """k, v [pages, Hkv, page, 128], with the heads or the places ahead."""
    shape = (pages, Hkv, page, 128) if order == "heads" else (pages, page, Hkv, 128)
    make = lambda: torch.randn(shape, generator=gen, device="cuda").to(dtype) if fill else torch.full(shape, 7.0, device="cuda", dtype=dtype)
    k, v = make(), make()
    return (k, v) if order == "heads" else (k.transpose(1, 2), v.transpose(1, 2))


def table_of(gen, lengths, page, width, shared=0):
    """A table of pages in no order, the first `shared` pages alike; what is behind a sequence's pages names none.  And how many pages there are."""
    B = len(lengths)
    total = shared + B * (width - shared) + 2
    order = torch.randperm(total, generator=gen, device="cuda").to(torch.int32)
    table = torch.full((B, width), -1, dtype=torch.int32, device="cuda")
    for b, N in enumerate(lengths):
        n = -(-N // page)
        table[b, :min(n, shared)] = order[:min(n, shared)]
        if n > shared:
            at = shared + b * (width - shared)
            table[b, shared:n] = order[at:at + n - shared]
    return table, total


def gathered(pages, table, b, N):
    """[Hkv, N, 128] of a sequence; positions without a page are zeros."""
    P, H, T, _ = pages.shape
    row = table[b, :-(-N // T)].long()
    there = (row >= 0) & (row < P)
    x = pages[row.clamp(0, P - 1)]
    x = torch.where(there[:, None, None, None], x, torch.zeros((), dtype=x.dtype, device=x.device))
    return x.transpose(0, 1).reshape(H, -1, 128)[:, :N]


def with_page(pages, table, b, N):
    P, _, T, _ = pages.shape
    row = table[b, :-(-N // T)]
    return ((row >= 0) & (row < P)).repeat_interleave(T)[:N]


def reference(q, k, v, table, n_of, N_of, scale, seen_of=None):
    """(outputs, tolerance) in 64 bits; rows behind a sequence's queries are NaN.  seen_of(b, KV head) narrows what the rows see: [n, N] or None.

    Tolerance of a channel, with A = sum_j p_j |v_j| (p the exact weights) and h half a step of the type: the weights' rounding h A, the final one h |o|; a score is
    off by the binary32 sum of 128 products, 2^-17 of sum |q||k| scale at most, which the exponential turns into twice that (numerator and sum) of A; the
    exponential, the binary32 sums, the rescaling and the joining of parts 2^-16 A.  In binary16 weights below 2^-14 of the largest are off by up to 2^-25
    absolute: that times the sum of |v| seen."""
    B, Hq, n_all, _ = q.shape
    G = Hq // k.shape[1]
    half = torch.finfo(q.dtype).eps / 2
    out = torch.full(q.shape, math.nan, device=q.device, dtype=torch.float64)
    tol = torch.zeros(q.shape, device=q.device, dtype=torch.float64)
    for b in range(B):
        n, N = n_of[b], N_of[b]
        if n == 0:
            continue
        if N == 0:
            out[b, :, :n] = 0
            continue
        p, j = N - n + torch.arange(n, device=q.device)[:, None], torch.arange(N, device=q.device)[None]
        K_all, V_all, paged = gathered(k, table, b, N), gathered(v, table, b, N), with_page(k, table, b, N)
        for h in range(Hq):
            seen = (j <= p) & paged
            if seen_of is not None:
                seen = seen & seen_of(b, h // G)
            K, V, Q = K_all[h // G].double(), V_all[h // G].double(), q[b, h, :n].double()
            x = torch.where(seen, Q @ K.t() * scale, -math.inf)
            most = x.amax(dim=1, keepdim=True)
            w = torch.where(seen, (x - torch.where(most == -math.inf, 0.0, most)).exp(), 0.0)
            total = w.sum(dim=1, keepdim=True)
            w = torch.where(total > 0, w / total, 0.0)
            o, A = torch.empty_like(Q), torch.empty_like(Q)
            if bool(torch.isfinite(V).all()) and bool(torch.isfinite(w).all()):
                o, A = w @ V, w @ V.abs()
            else:
                for i in range(n):
                    s = seen[i]
                    o[i] = (w[i, s][:, None] * V[s]).sum(dim=0)
                    A[i] = (w[i, s][:, None] * V[s].abs()).sum(dim=0)
            size = torch.where(seen, Q.abs() @ K.abs().t() * scale, 0.0).nan_to_num(0, 0, 0).amax(dim=1, keepdim=True)
            t = A * (half + 2 * 2.0 ** -17 * size + 2.0 ** -16) + half * o.abs()
            if q.dtype == torch.float16:
                t = t + 2.0 ** -25 * (1 + seen.double() @ V.abs().nan_to_num(0, 0, 0))
            out[b, h, :n], tol[b, h, :n] = o, t
    return out, tol


def compare(got, exact, tol, n_of):
    """Everything asked for within its tolerance, not finite where the reference is not, rows behind the queries as they were (7)."""
    asked = torch.zeros(got.shape, dtype=torch.bool, device="cuda")
    for b, n in enumerate(n_of):
        asked[b, :, :n] = True
    assert bool((got[~asked] == 7.0).all()), "rows behind the queries were written"
    finite = asked & torch.isfinite(exact)
    assert bool((~torch.isfinite(got))[asked & ~torch.isfinite(exact)].all())
    off = ((got.double() - exact).abs() - tol)[finite]
    assert bool(torch.isfinite(got[finite]).all()) and (off.numel() == 0 or off.max().item() <= 0), off.max().item()


def ints(x):
    return None if x is None else torch.tensor(x, dtype=torch.int32, device="cuda")


def scratch_of(need):
    return torch.full((need,), 255, dtype=torch.uint8, device="cuda") if need else None


def attend(cache, q, kv_tokens, shared=0, n_of=None, N_of=None, sm_scale=0.0, out=None, stream=None):
    out = torch.full(q.shape, 7.0, device="cuda", dtype=q.dtype) if out is None else out
    scratch = scratch_of(binding.paged_scratch(cache, q.shape[0], q.shape[1], q.shape[2], kv_tokens, shared))
    binding.paged_attend(cache, q, out, kv_tokens, shared, ints(n_of), ints(N_of), sm_scale, scratch, stream)
    return out
