"""The 16-bit paged cache around the cache's calls, as cases that can be timed and compared: appending to it with the rotation
on the way ("append"), attention of a batch that shares a prefix ("attend"), and sparse attention over blocks chosen by a cheap
score ("blocks").

A paged cache holds the keys and values of a layer in pages of P places: k, v [pages, KV head, place, 128] (or with the places
ahead of the heads); table[b][i] is the page of positions i * P .. i * P + P - 1 of sequence b, an entry outside the pages is none.  bounds [pages, KV
head, 2, 128] are the least and the largest key of a page, channel by channel.

append: token t < n of sequence b goes to position starts[b] + t; its key is turned by the rotary angles of that position, its value goes
through, its queries are turned into an array of their own.  A page's bounds begin anew with its place 0.

attend: row i of a sequence with n queries and N cached tokens stands at position p = N - n + i and sees the positions j <= p.  The
first shared // P pages of all sequences are the same.

blocks: a block is a page.  Of the blocks up to a row's own (p // P), the first `first`, the last `recent` (its own among them) and
the `top` others of the largest score are listed in ascending order (-1 behind them); a block's score for a KV head is the
largest of its query heads' max(q, 0) . kmax + min(q, 0) . kmin, the lower block first among equals.  The row then sees the positions j <= p of
the listed blocks.

Shapes are those of the benchmark's configurations (32 heads of 128 channels, alone or on 8 KV heads, 2k to 131k tokens, batches up
to 16) or generic ones.
"""
import math

import torch

own = False
D = 128
DTYPES = {"fp16": torch.float16, "bf16": torch.bfloat16}
BLOCK = 1 << 28        # scores, or gathered channels, that the plain forms hold at a time


def _case(name, **c):
    return dict(c, name=name) if name else c


def _append(name, batch, tokens, q_heads, kv_heads, page, order, bounds, rotary_dim, layout, scaling, base, first, ragged, dtype):
    return _case(name, op="append", batch=batch, tokens=tokens, q_heads=q_heads, kv_heads=kv_heads, page=page, order=order, bounds=bounds,
                 rotary_dim=rotary_dim, layout=layout, scaling=scaling, base=base, first=first, ragged=ragged, dtype=dtype)


def _attend(name, batch, q_tokens, shared, more, q_heads, kv_heads, page, order, ragged, dtype):
    return _case(name, op="attend", batch=batch, q_tokens=q_tokens, shared=shared, more=more, q_heads=q_heads, kv_heads=kv_heads, page=page,
                 order=order, ragged=ragged, dtype=dtype)


def _blocks(name, batch, q_tokens, kv_tokens, q_heads, kv_heads, page, order, top, first, recent, ragged, dtype):
    return _case(name, op="blocks", batch=batch, q_tokens=q_tokens, kv_tokens=kv_tokens, q_heads=q_heads, kv_heads=kv_heads, page=page,
                 order=order, top=top, first=first, recent=recent, ragged=ragged, dtype=dtype)


def listed():
    return [
        # a step of a batch, every sequence at a length of its own: a call's latency
        _append("append_step_16", 16, 1, 32, 8, 64, "heads", True, 128, "half", "none", 5.0e5, 2000, False, "bf16"),
        # a whole prompt of a model whose positions are scaled by wavelength: the most bytes of an append
        _append("append_prompt_32k", 1, 32768, 32, 8, 16, "heads", True, 128, "half", "bands", 5.0e5, 0, False, "bf16"),
        # parts of prompts of odd lengths behind what is cached, neighbouring channels paired, half of the head, no bounds kept
        _append("append_ragged_5", 5, 3001, 32, 32, 32, "places", False, 64, "interleaved", "none", 1.0e4, 700, True, "fp16"),
        # three samples of one short prompt, a head to each KV head: latency again
        _attend("attend_step_short", 3, 1, 1000, 200, 32, 32, 16, "heads", True, "fp16"),
        # a full batch behind one long system prompt: the prefix is read once
        _attend("attend_step_64_prefix_32k", 64, 1, 32768, 1024, 32, 8, 64, "heads", True, "bf16"),
        # the two rows of each sequence's step, long turns of their own behind a prefix that ends inside a page
        _attend("attend_step_16_prefix_8k", 16, 2, 8197, 4000, 64, 8, 32, "places", True, "fp16"),
        # nothing shared: a batch of sequences of every length, the smallest pages, the most bytes
        _attend("attend_step_batch16", 16, 1, 0, 32768, 32, 8, 16, "heads", True, "bf16"),
        # the questions behind a shared document, as prompts: the most products
        _attend("attend_chunks_prefix_16k", 8, 256, 16384, 600, 32, 8, 64, "heads", True, "bf16"),
        # the two rows of a decode step, a head to each KV head
        _blocks("blocks_step_16k", 1, 2, 16384, 32, 32, 16, "heads", 32, 1, 4, False, "fp16"),
        # a batch of sequences of every length takes a step
        _blocks("blocks_step_batch16", 16, 1, 32768, 32, 8, 64, "heads", 32, 1, 2, True, "bf16"),
        # one long context in small blocks: the scores are most of it
        _blocks("blocks_step_131k", 1, 1, 131072, 32, 8, 32, "places", 64, 4, 8, False, "bf16"),
        # a part of a prompt, every token with blocks of its own
        _blocks("blocks_chunk_128", 2, 128, 20011, 64, 8, 64, "heads", 16, 1, 2, True, "bf16"),
    ]


def _spread(rng, low, high):
    return max(low, min(high, round(low * (high / low) ** rng.random())))


def draw(rng):
    op = rng.choice(["append", "attend", "attend", "blocks", "blocks"])
    q_heads, kv_heads = rng.choice([(32, 32), (32, 8), (64, 8), (16, 8), (8, 1), (5, 5)])
    page, order, dtype = rng.choice([16, 32, 64, 64, 128, 256]), rng.choice(["heads", "heads", "places"]), rng.choice(["fp16", "bf16"])
    batch = rng.choice([1, 2, 3, 5, 16])
    if op == "append":
        batch = rng.choice([batch, 64])
        tokens = min(_spread(rng, 1, max(1, 32768 * 48 // (batch * (q_heads + 2 * kv_heads)))), 32768)
        return _append(None, batch, tokens, q_heads, kv_heads, page, order, rng.random() < 0.6, rng.choice([128, 128, 64, 32, 96, 16]),
                       rng.choice(["half", "half", "interleaved"]), rng.choice(["none", "none", "linear", "bands"]), rng.choice([1.0e4, 5.0e5, 1.0e6]),
                       rng.choice([0, _spread(rng, 1, min(4000, 1_000_000 // (batch * kv_heads)))]), rng.random() < 0.5, dtype)
    if op == "attend":
        batch = rng.choice([batch, 32, 64])
        pairs = 1_200_000 // kv_heads                                 # places of the pool: 0.6 GB
        shared = rng.choice([0, 1, 1]) * _spread(rng, 50, min(65536, 1_000_000 // kv_heads))
        more = _spread(rng, 1, max(1, min(32768, pairs // batch)))
        if rng.random() < 0.7:
            q_tokens = rng.choice([1, 1, 1, 2, 2, 3, 4])
            more = max(more, q_tokens)
            shared = min(shared, (1 << 29) // (batch * q_tokens * q_heads))
        else:
            q_tokens = _spread(rng, 2, 512)
            more = max(min(more, 4096), q_tokens)
            batch = max(1, min(batch, (1 << 28) // (q_tokens * q_heads * more)))
            shared = min(shared, (3 << 28) // (batch * q_tokens * q_heads))
        return _attend(None, batch, q_tokens, shared, more, q_heads, kv_heads, page, order, rng.random() < 0.6, dtype)
    q_tokens = rng.choice([1, 1, 1, 2, 2, 4, _spread(rng, 5, 128)])
    kv_tokens = max(q_tokens, _spread(rng, 100, min(131072, (1 << 21) // (batch * kv_heads))))
    top = _spread(rng, 1, max(1, 2048 // page))
    if q_tokens > 4:
        batch = min(batch, 2)
    return _blocks(None, batch, q_tokens, kv_tokens, q_heads, kv_heads, page, order, top, rng.choice([0, 1, 1, 4]), rng.choice([0, 1, 2, 2, 8]),
                   rng.random() < 0.5, dtype)


# ---- what the cases have in hand -------------------------------------------------------------------------------------

def _pool(case, gen, pages, fill):
    """k, v [pages, KV head, place, 128]; fill: with keys that have a few large channels and a direction to each page."""
    h, p, dtype = case["kv_heads"], case["page"], DTYPES[case["dtype"]]
    shape = (pages, h, p, D) if case["order"] == "heads" else (pages, p, h, D)
    k, v = (torch.zeros(shape, device="cuda", dtype=dtype) for _ in range(2))
    if case["order"] == "places":
        k, v = k.transpose(1, 2), v.transpose(1, 2)
    if fill:
        k.normal_(generator=gen)
        v.normal_(generator=gen)
        large = torch.randint(0, D, (h, 2), generator=gen, device="cuda")
        k.mul_(torch.ones((h, D), device="cuda").scatter_(1, large, 4.0)[:, None].to(dtype))
        k.add_(torch.randn((pages, h, 1, D), generator=gen, device="cuda").mul_(0.5).to(dtype))
    return k, v


def _table(gen, shared_pages, pages_of, page_most):
    """Pages in no order, the first shared_pages the same for all; entries behind a sequence's pages are none.  As many pages as sequences of
    page_most pages would take, and a few that nobody has."""
    total = shared_pages + len(pages_of) * (page_most - shared_pages) + 3
    order = torch.randperm(total, generator=gen, device="cuda").to(torch.int32)
    table = torch.full((len(pages_of), page_most), -1, dtype=torch.int32, device="cuda")
    at = shared_pages
    for b, n in enumerate(pages_of):
        alike = min(n, shared_pages)
        table[b, :alike] = order[:alike]
        table[b, alike:n] = order[at:at + n - alike]
        at += n - alike
    return table, total


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _lengths(case, gen, most, least):
    """Of a ragged batch: the first sequence the longest, the others of every length."""
    B = case["batch"]
    if not case["ragged"]:
        return [most] * B
    part = torch.rand(B, generator=gen, device="cuda").tolist()
    return [most] + [least + int(r * (most - least)) for r in part[1:]]


# ---- appending -------------------------------------------------------------------------------------------------------

FACTOR, ORIGINAL, BANDS = 8.0, 8192, (1.0, 4.0)


def _frequencies(case):
    """Angle per position of every pair of channels, in 64 bits."""
    d = case["rotary_dim"]
    f = case["base"] ** (-2 * torch.arange(d // 2, dtype=torch.float64, device="cuda") / d)
    if case["scaling"] == "linear":
        return f / FACTOR
    if case["scaling"] == "bands":
        keep = ((ORIGINAL * f / (2 * math.pi) - BANDS[0]) / (BANDS[1] - BANDS[0])).clamp(0, 1)
        return keep * f + (1 - keep) * f / FACTOR
    return f


def _append_prepare(case, gen):
    B, L, Hq, Hkv, P = case["batch"], case["tokens"], case["q_heads"], case["kv_heads"], case["page"]
    dtype = DTYPES[case["dtype"]]
    s = {"case": case, "x": torch.randn((B, L, Hq + 2 * Hkv, D), generator=gen, device="cuda", dtype=dtype).transpose(1, 2)}
    s["starts_of"] = [int(r * case["first"]) for r in torch.rand(B, generator=gen, device="cuda").tolist()]
    s["lengths_of"] = _lengths(case, gen, L, 1)
    ends = [a + n for a, n in zip(s["starts_of"], s["lengths_of"])]
    s["starts"], s["lengths"] = _ints(s["starts_of"]), _ints(s["lengths_of"])
    s["table"], pages = _table(gen, 0, [-(-e // P) for e in ends], -(-(case["first"] + L) // P))
    s["k"], s["v"] = _pool(case, gen, pages, False)
    s["bounds"] = torch.zeros((pages, Hkv, 2, D), device="cuda", dtype=dtype) if case["bounds"] else None
    s["q"] = torch.zeros((B, Hq, L, D), device="cuda", dtype=dtype)
    if own:
        from paper_2503_16163_amd import binding
        layout = {"half": binding.ROTARY_HALF, "interleaved": binding.ROTARY_INTERLEAVED}[case["layout"]]
        scaling = {"none": binding.ROTARY_UNSCALED, "linear": binding.ROTARY_LINEAR, "bands": binding.ROTARY_BANDS}[case["scaling"]]
        s["plan"] = binding.rotary_plan(case["rotary_dim"], case["base"], layout, scaling, FACTOR, ORIGINAL, *BANDS)
        s["cache"] = binding.Pages(s["k"], s["v"], s["table"], s["bounds"])
    return s


def _append_out(s):
    out = {"q": s["q"], "k": s["k"], "v": s["v"]}
    return dict(out, bounds=s["bounds"]) if s["case"]["bounds"] else out


def _split(s):
    Hq, Hkv = s["case"]["q_heads"], s["case"]["kv_heads"]
    return s["x"][:, :Hq], s["x"][:, Hq:Hq + Hkv], s["x"][:, Hq + Hkv:]


def _append_own(s):
    from paper_2503_16163_amd import binding
    q, k, v = _split(s)
    binding.paged_append(s["cache"], s["plan"], k, v, q, s["q"], starts=s["starts"], lengths=s["lengths"] if s["case"]["ragged"] else None)
    return _append_out(s)


def _turned(case, x, cos, sin):
    d = case["rotary_dim"]
    if case["layout"] == "half":
        a, b = x[..., :d // 2], x[..., d // 2:d]
        return torch.cat([a * cos - b * sin, b * cos + a * sin, x[..., d:]], dim=-1)
    a, b = x[..., 0:d:2], x[..., 1:d:2]
    return torch.cat([torch.stack([a * cos - b * sin, b * cos + a * sin], dim=-1).flatten(-2), x[..., d:]], dim=-1)


def _append_plain(s):
    case, P = s["case"], s["case"]["page"]
    q, k, v = _split(s)
    f = _frequencies(case)
    for b, (start, n) in enumerate(zip(s["starts_of"], s["lengths_of"])):
        at = start + torch.arange(n, device="cuda")
        angle = at.double()[:, None] * f                              # far positions need the 64 bits
        cos, sin = angle.cos().float(), angle.sin().float()
        s["q"][b, :, :n] = _turned(case, q[b, :, :n].float(), cos, sin).to(s["q"].dtype)
        turned = _turned(case, k[b, :, :n].float(), cos, sin).to(s["k"].dtype)
        pages, places = s["table"][b][at // P].long(), at % P
        s["k"][pages, :, places] = turned.transpose(0, 1)
        s["v"][pages, :, places] = v[b, :, :n].transpose(0, 1)
        if case["bounds"]:
            fresh = s["table"][b, -(-start // P):-(-(start + n) // P)].long()
            s["bounds"][fresh, :, 0] = math.inf
            s["bounds"][fresh, :, 1] = -math.inf
            index = pages[:, None, None].expand(n, case["kv_heads"], D)
            low, high = s["bounds"][:, :, 0].float(), s["bounds"][:, :, 1].float()
            rows = turned.transpose(0, 1).float()
            s["bounds"][:, :, 0] = low.scatter_reduce(0, index, rows, "amin")
            s["bounds"][:, :, 1] = high.scatter_reduce(0, index, rows, "amax")
    return _append_out(s)


def _append_exact(case, s):
    # every pair of channels as a complex number times e^(i angle), page by page
    P, d, Hkv = case["page"], case["rotary_dim"], case["kv_heads"]
    turns = _frequencies(case)
    q, k, v = _split(s)
    first, second = (range(0, d // 2), range(d // 2, d)) if case["layout"] == "half" else (range(0, d, 2), range(1, d, 2))
    first, second = list(first), list(second)
    out = {"q": s["q"].double(), "k": s["k"].double().contiguous(), "v": s["v"].double().contiguous()}
    if case["bounds"]:
        out["bounds"] = s["bounds"].double()
    table = s["table"].tolist()
    for b, (start, n) in enumerate(zip(s["starts_of"], s["lengths_of"])):
        angle = (start + torch.arange(n, dtype=torch.float64, device="cuda"))[:, None] * turns
        turn = torch.polar(torch.ones_like(angle), angle)

        def rotated(x):
            y = x.double().contiguous()
            z = torch.complex(y[..., first], y[..., second]) * turn
            y[..., first], y[..., second] = z.real, z.imag
            return y
        out["q"][b, :, :n] = rotated(q[b, :, :n])
        keys, values = rotated(k[b, :, :n]), v[b, :, :n].double()
        for i in range(start // P, (start + n - 1) // P + 1):
            lo, hi = max(start, i * P), min(start + n, i * P + P)
            page = table[b][i]
            here = keys[:, lo - start:hi - start]
            out["k"][page, :, lo - i * P:hi - i * P] = here
            out["v"][page, :, lo - i * P:hi - i * P] = values[:, lo - start:hi - start]
            if case["bounds"]:
                low, high = here.amin(dim=1), here.amax(dim=1)
                if lo > i * P:                                        # what the page's earlier places left
                    low, high = torch.minimum(low, out["bounds"][page, :, 0]), torch.maximum(high, out["bounds"][page, :, 1])
                out["bounds"][page, :, 0], out["bounds"][page, :, 1] = low, high
    return out


# ---- attention of a batch that shares a prefix -----------------------------------------------------------------------

def _attend_prepare(case, gen):
    B, n, Hq, P = case["batch"], case["q_tokens"], case["q_heads"], case["page"]
    s = {"case": case}
    s["cached"] = [case["shared"] + m for m in _lengths(case, gen, case["more"], min(n, case["more"]))]
    s["most"] = case["shared"] + case["more"]
    s["table"], pages = _table(gen, case["shared"] // P, [-(-c // P) for c in s["cached"]], -(-s["most"] // P))
    s["k"], s["v"] = _pool(case, gen, pages, True)
    s["q"] = torch.randn((B, n, Hq, D), generator=gen, device="cuda", dtype=DTYPES[case["dtype"]]).transpose(1, 2)
    s["out"] = torch.zeros_like(s["q"])
    s["kv_lengths"] = _ints(s["cached"])
    if own:
        from paper_2503_16163_amd import binding
        s["cache"] = binding.Pages(s["k"], s["v"], s["table"])
        need = binding.paged_scratch(s["cache"], B, Hq, n, s["most"], case["shared"])
        s["scratch"] = torch.empty(need, dtype=torch.uint8, device="cuda") if need else None
    return s


def _attend_own(s):
    from paper_2503_16163_amd import binding
    binding.paged_attend(s["cache"], s["q"], s["out"], s["most"], s["case"]["shared"], kv_lengths=s["kv_lengths"], scratch=s["scratch"])
    return s["out"]


def _sequence(s, b, N):
    """Keys and values of a sequence's N positions: [KV head, N, 128]."""
    P, H = s["case"]["page"], s["case"]["kv_heads"]
    pages = s["table"][b, :-(-N // P)].long()
    return (x[pages].transpose(0, 1).reshape(H, -1, D)[:, :N] for x in (s["k"], s["v"]))


def _attend_plain(s):
    case, scale = s["case"], 1 / math.sqrt(D)
    n, Hkv, G = case["q_tokens"], case["kv_heads"], case["q_heads"] // case["kv_heads"]
    for b, N in enumerate(s["cached"]):
        k, v = (x.float() for x in _sequence(s, b, N))
        k = k.transpose(1, 2).contiguous()
        step = max(1, min(n, BLOCK // (case["q_heads"] * N)))
        for i in range(0, n, step):
            m = min(step, n - i)
            p = torch.arange(N - n + i, N - n + i + m, device="cuda")[:, None]
            hidden = torch.arange(N, device="cuda") > p
            q = s["q"][b, :, i:i + m].float().reshape(Hkv, G * m, D)
            x = torch.matmul(q, k).view(Hkv, G, m, N).mul_(scale)
            x.masked_fill_(hidden, -math.inf)
            x = x.sub_(x.amax(dim=-1, keepdim=True)).exp_()
            total = x.sum(dim=-1)
            o = torch.matmul(x.view(Hkv, G * m, N), v).view(Hkv, G, m, D) / total[..., None]
            s["out"][b, :, i:i + m] = o.reshape(case["q_heads"], m, D)
    return s["out"]


def _attend_exact(case, s):
    # head by head in 64 bits, all of a sequence's rows at once
    n, Hq, Hkv = case["q_tokens"], case["q_heads"], case["kv_heads"]
    out = torch.zeros((case["batch"], n, Hq, D), device="cuda", dtype=torch.float64).transpose(1, 2)
    for b, N in enumerate(s["cached"]):
        at, pos = torch.arange(N, device="cuda"), N - n + torch.arange(n, device="cuda").view(-1, 1)
        keys, values = _sequence(s, b, N)
        for h in range(Hkv):
            kh, vh = keys[h].double(), values[h].double()
            for g in range(h * (Hq // Hkv), (h + 1) * (Hq // Hkv)):
                x = torch.where(at <= pos, s["q"][b, g].double() @ kh.t() / math.sqrt(D), -math.inf)
                out[b, g] = torch.softmax(x, dim=1) @ vh
    return out


# ---- sparse attention over chosen blocks -----------------------------------------------------------------------------

def _blocks_prepare(case, gen):
    B, n, Hq, Hkv, P = case["batch"], case["q_tokens"], case["q_heads"], case["kv_heads"], case["page"]
    s = {"case": case, "cached": _lengths(case, gen, case["kv_tokens"], min(n, case["kv_tokens"]))}
    s["table"], pages = _table(gen, 0, [-(-c // P) for c in s["cached"]], -(-case["kv_tokens"] // P))
    s["k"], s["v"] = _pool(case, gen, pages, True)
    s["bounds"] = torch.stack([s["k"].amin(dim=2), s["k"].amax(dim=2)], dim=2).contiguous()
    s["q"] = torch.randn((B, n, Hq, D), generator=gen, device="cuda", dtype=DTYPES[case["dtype"]]).transpose(1, 2)
    s["out"] = torch.zeros_like(s["q"])
    s["blocks"] = torch.full((B, Hkv, n, case["first"] + case["top"] + case["recent"]), -1, dtype=torch.int32, device="cuda")
    s["kv_lengths"] = _ints(s["cached"])
    if own:
        from paper_2503_16163_amd import binding
        s["cache"] = binding.Pages(s["k"], s["v"], s["table"], s["bounds"])
        need = binding.block_scratch(s["cache"], B, Hq, n, case["kv_tokens"], case["top"], case["first"], case["recent"])
        s["scratch"] = torch.empty(need, dtype=torch.uint8, device="cuda") if need else None
    return s


def _blocks_own(s):
    from paper_2503_16163_amd import binding
    c = s["case"]
    binding.block_select(s["cache"], s["q"], s["blocks"], c["kv_tokens"], c["top"], c["first"], c["recent"], kv_lengths=s["kv_lengths"], scratch=s["scratch"])
    binding.block_attend(s["cache"], s["q"], s["out"], s["blocks"], c["kv_tokens"], kv_lengths=s["kv_lengths"], scratch=s["scratch"])
    return {"blocks": s["blocks"], "out": s["out"]}


def _blocks_plain(s):
    case, P, scale = s["case"], s["case"]["page"], 1 / math.sqrt(D)
    n, Hkv, G = case["q_tokens"], case["kv_heads"], case["q_heads"] // case["kv_heads"]
    slots = case["first"] + case["top"] + case["recent"]
    s["blocks"].fill_(-1)
    for b, N in enumerate(s["cached"]):
        have = -(-N // P)
        pages = s["table"][b, :have].long()
        least, most = (s["bounds"][pages, :, i].double().permute(1, 2, 0).contiguous() for i in (0, 1))       # [KV head, 128, block]
        q = s["q"][b].double().reshape(Hkv, G * n, D)
        # 64 bits: scores next to each other decide
        score = (torch.matmul(q.clamp(min=0), most) + torch.matmul(q.clamp(max=0), least)).view(Hkv, G, n, have).amax(dim=1)
        p = torch.arange(N - n, N, device="cuda")[:, None]
        block, last = torch.arange(have, device="cuda"), p // P
        kept = ((block < case["first"]) | (block > last - case["recent"])) & (block <= last)
        rest = torch.where(kept | (block > last), -math.inf, score)
        value, index = rest.sort(dim=-1, descending=True, stable=True)
        value, index = value[..., :case["top"]], index[..., :case["top"]]
        chosen = torch.zeros((Hkv, n, have), dtype=torch.bool, device="cuda").scatter_(2, index, value > -math.inf) | kept
        names = torch.where(chosen, block, have).sort(dim=-1)[0][..., :slots]
        s["blocks"][b, ..., :names.shape[-1]] = torch.where(names < have, names, -1).to(torch.int32)
        step = max(1, BLOCK // (Hkv * slots * P * D))
        for i in range(0, n, step):
            listed_ = s["blocks"][b, :, i:i + step].long()                                                   # [KV head, m, slot]
            m = listed_.shape[1]
            at = (listed_[..., None] * P + torch.arange(P, device="cuda")).flatten(2)
            seen = (listed_ >= 0)[..., None].expand(-1, -1, -1, P).flatten(2) & (at <= p[i:i + m])
            page = s["table"][b][listed_.clamp(min=0)].long().clamp(min=0)
            head = torch.arange(Hkv, device="cuda")[:, None, None]
            k, v = (x[page, head].flatten(2, 3).float() for x in (s["k"], s["v"]))                            # [KV head, m, slot * P, 128]
            qs = s["q"][b, :, i:i + m].float().view(Hkv, G, m, D).transpose(1, 2)
            x = torch.matmul(qs, k.transpose(2, 3).contiguous()).mul_(scale)                                  # [KV head, m, G, slot * P]
            x.masked_fill_(~seen[:, :, None], -math.inf)
            x = x.sub_(x.amax(dim=-1, keepdim=True)).exp_()
            o = torch.matmul(x, v) / x.sum(dim=-1, keepdim=True)
            s["out"][b, :, i:i + m] = o.transpose(1, 2).reshape(case["q_heads"], m, D)
    return {"blocks": s["blocks"], "out": s["out"]}


def _blocks_exact(case, s):
    # head by head: the larger of the two products channel by channel; attention over all that is cached, what is not listed hidden
    P, n, Hq, Hkv = case["page"], case["q_tokens"], case["q_heads"], case["kv_heads"]
    G = Hq // Hkv
    blocks = torch.full_like(s["blocks"], -1)
    out = torch.zeros((case["batch"], n, Hq, D), device="cuda", dtype=torch.float64).transpose(1, 2)
    for b, N in enumerate(s["cached"]):
        have = -(-N // P)
        pages = s["table"][b, :have].long()
        keys, values = _sequence(s, b, N)
        pos = (N - n + torch.arange(n, device="cuda"))[:, None]
        number, mine = torch.arange(have, device="cuda"), pos // P
        for h in range(Hkv):
            low, high = s["bounds"][pages, h, 0].double(), s["bounds"][pages, h, 1].double()
            best = torch.full((n, have), -math.inf, device="cuda", dtype=torch.float64)
            step = max(1, BLOCK // 4 // (have * D))
            for g in range(h * G, (h + 1) * G):
                for i in range(0, n, step):
                    q = s["q"][b, g, i:i + step].double()[:, None]
                    best[i:i + step] = torch.maximum(best[i:i + step], torch.maximum(q * low, q * high).sum(dim=-1))
            best[number > mine] = -math.inf
            best[(number < case["first"]) | ((number <= mine) & (number > mine - case["recent"]))] = math.inf
            best[number > mine] = -math.inf
            forced = (best == math.inf).sum(dim=1)
            count = torch.minimum(forced + case["top"], mine[:, 0] + 1)
            order = torch.argsort(-best, dim=1, stable=True)
            rank = torch.empty_like(order).scatter_(1, order, number.expand(n, -1).contiguous())
            taken = rank < count[:, None]
            for i, row in enumerate(taken.cpu()):
                ids = row.nonzero()[:, 0].to(torch.int32)
                blocks[b, h, i, :len(ids)] = ids.cuda()
            hidden = ~(taken.repeat_interleave(P, dim=1)[:, :N] & (torch.arange(N, device="cuda") <= pos))
            kh, vh = keys[h].double(), values[h].double()
            for g in range(h * G, (h + 1) * G):
                x = (s["q"][b, g].double() @ kh.t() / math.sqrt(D)).masked_fill(hidden, -math.inf)
                out[b, g] = torch.softmax(x, dim=1) @ vh
    return {"blocks": blocks, "out": out}


# ---- what the tools call ---------------------------------------------------------------------------------------------

_PREPARE = {"append": _append_prepare, "attend": _attend_prepare, "blocks": _blocks_prepare}
_PLAIN = {"append": _append_plain, "attend": _attend_plain, "blocks": _blocks_plain}
_OWN = {"append": _append_own, "attend": _attend_own, "blocks": _blocks_own}
_EXACT = {"append": _append_exact, "attend": _attend_exact, "blocks": _blocks_exact}


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return _PREPARE[case["op"]](case, gen)


def run(state):
    return (_OWN if own else _PLAIN)[state["case"]["op"]](state)


def exact(case, seed):
    return _EXACT[case["op"]](case, prepare(case, seed))


def work(case):
    B, Hq, Hkv, P = case["batch"], case["q_heads"], case["kv_heads"], case["page"]
    part = (1 + (B - 1) * 0.5) / B if case["ragged"] else 1.0       # of a ragged batch's lengths half on average
    if case["op"] == "append":
        tokens = B * case["tokens"] * part
        kept = -(-tokens // P) * Hkv * 2 * D * 2 if case["bounds"] else 0
        return {"bytes": tokens * (Hq + 2 * Hkv) * 2 * D * 2 + kept, "flops": tokens * (Hq + Hkv) * 3 * case["rotary_dim"]}
    n = case["q_tokens"]
    rows = 4 * D * B * Hq * n                                       # bytes of q and out
    if case["op"] == "attend":
        more = case["more"] * part
        seen = case["shared"] + max(more - (n - 1) / 2, 1)
        return {"bytes": 4 * D * Hkv * (case["shared"] + B * more) + rows, "flops": 4 * D * B * Hq * n * seen}
    cached, slots = case["kv_tokens"] * part, case["first"] + case["top"] + case["recent"]
    seen = min(slots * P, cached)
    pairs = B * Hkv * min(n * seen, cached)                         # rows of a part of a prompt share what they read
    scores = B * Hkv * cached / P
    return {"bytes": 4 * D * (pairs + scores) + rows + 4 * B * Hkv * n * slots, "flops": 4 * D * B * Hq * n * (seen + cached / P)}
