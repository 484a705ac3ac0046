"""Timed operators next to a paged KV cache: several rows over one context, drafted tokens, and the pages worth reading.

* ``shared``   attention of the rows of a group that share the first positions of their contexts (a batch with one system
               prompt, the beams of a search, the drafted tokens of one sequence): the shared positions are read once for all
* ``verify``   which of the tokens that a cheaper model drafted are kept, and the token behind them, from the logits of the
               target, those of the draft, and given random numbers
* ``bound``    the smallest and the largest key of every page, dimension by dimension
* ``pick``     the pages of a long context whose bounds promise the largest scores, for every query and kv head
* ``picked``   attention of one new token per sequence over the pages that were picked for each kv head

A pool of pages is ``k, v [layer][page][kv head][row of the page][head_dim]``, 8-bit pools with one fp32 scale for each row;
a table gives for every sequence the pages of its positions in order.

Shapes are those of the repository's own models (16 or 32 query and 8 kv heads of 128, a vocabulary of 151936) and generic
ones around them.
"""
import math

import numpy as np
import torch

own = False

DEVICE = "cuda:0"
TORCH = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16, "i8": torch.int8, "e4m3": torch.float8_e4m3fn}
BYTES = {"f32": 4, "bf16": 2, "f16": 2, "i8": 1, "e4m3": 1}
TOP = {"i8": 127.0, "e4m3": 448.0}     # largest magnitude that a stored value stands for, before its scale
VOCAB = 151936


def _bound_type(store):
    """Bounds are held in the pool's own type, those of 8-bit pools in bf16, rounded outwards."""
    return "bf16" if store in TOP else store


def listed():
    return [
        # one search of four beams early in a chat (launch latency)
        dict(name="shared-w4-c300", op="shared", store="bf16", q="bf16", groups=1, width=4, kv_heads=8, group=2, head_dim=128, page_tokens=16,
             prefix_least=304, prefix=304, behind_least=1, behind=16, drafts=False, strided=False),
        # a server's batch behind one long system prompt
        dict(name="shared-w64-c16384", op="shared", store="bf16", q="bf16", groups=1, width=64, kv_heads=8, group=4, head_dim=128, page_tokens=64,
             prefix_least=16384, prefix=16384, behind_least=0, behind=500, drafts=False, strided=False),
        # four drafted tokens and the one before them, of several users, in an 8-bit cache; queries as the projection leaves them
        dict(name="shared-drafts-i8", op="shared", store="i8", q="f32", groups=4, width=5, kv_heads=8, group=4, head_dim=128, page_tokens=16,
             prefix_least=333, prefix=4100, behind_least=0, behind=0, drafts=True, strided=True),
        # one user's draft found in the prompt (no probabilities of its own), fp32 logits as the model leaves them
        dict(name="verify-n1-k4", op="verify", logits="f32", n=1, k=4, vocab=VOCAB, drafter=False, temperature=1.0, ragged=False),
        # a server's batch, drafts of different lengths, a mixture of sampled and greedy sequences
        dict(name="verify-n16-k5-ragged", op="verify", logits="f32", n=16, k=5, vocab=VOCAB, drafter=True, temperature=-1.0, ragged=True),
        # a large batch in 16 bits
        dict(name="verify-bf16-n64-k7", op="verify", logits="bf16", n=64, k=7, vocab=VOCAB, drafter=True, temperature=0.8, ragged=False),
        # a full prompt has gone into pages: the bounds of all of them
        dict(name="bound-bf16-p16384", op="bound", store="bf16", n_seqs=1, kv_heads=8, head_dim=128, page_tokens=16, shortest=16384, longest=16384, new=0),
        # one decode step of a batch: the pages that got a row
        dict(name="bound-i8-b48-step", op="bound", store="i8", n_seqs=48, kv_heads=8, head_dim=128, page_tokens=32, shortest=100, longest=3000, new=1),
        # one user on a book
        dict(name="pick-b1-c131072", op="pick", store="bf16", q="bf16", n_seqs=1, kv_heads=8, group=4, head_dim=128, page_tokens=16, shortest=131072, longest=131072,
             keep=256, first=1, last=2),
        # a server's batch of contexts of different lengths, in an 8-bit cache
        dict(name="pick-b16-ragged", op="pick", store="e4m3", q="f32", n_seqs=16, kv_heads=8, group=4, head_dim=128, page_tokens=32, shortest=1000, longest=16384,
             keep=64, first=1, last=1),
        # ... and the attention over what was picked for them
        dict(name="picked-b1-k256", op="picked", store="bf16", q="bf16", n_seqs=1, kv_heads=8, group=4, head_dim=128, page_tokens=16, shortest=131072, longest=131072, keep=256),
        dict(name="picked-b16-e4m3", op="picked", store="e4m3", q="f32", n_seqs=16, kv_heads=8, group=4, head_dim=128, page_tokens=32, shortest=1000, longest=16384, keep=64),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _cost(case):
    w = work(case)
    return w["bytes"] / 6e12 + w["flops"] / 5e14


def draw(rng):
    most = max(_cost(c) for c in listed())
    while True:
        op = rng.choice(["shared", "shared", "shared", "verify", "verify", "bound", "pick", "pick", "picked"])
        store = rng.choice(["bf16", "f16", "i8", "e4m3", "bf16", "f32"])
        shape = dict(store=store, kv_heads=rng.choice([1, 2, 3, 4, 5, 8, 8, 16]), head_dim=rng.choice([64, 128, 128]),
                     page_tokens=rng.choice([8, 16, 16, 24, 32, 64, 128]))
        queries = dict(q=rng.choice(["f32", "bf16", "f16"]), group=rng.choice([1, 2, 3, 4, 5, 8, 16]))
        if op == "shared":
            drafts = rng.random() < 0.4
            longest, width = _log_uniform(rng, 1, 32768), _log_uniform(rng, 1, 16 if drafts else 100)
            longest = max(longest, width)
            behind = 0 if drafts else rng.choice([0, rng.randint(1, 40), rng.randint(1, 700)])
            c = dict(op=op, **shape, **queries, groups=rng.choice([1, 1, 2, 3, 6]), width=width, prefix_least=max(width, longest // rng.choice([1, 1, 3])), prefix=longest,
                     behind_least=behind // rng.choice([1, 3]), behind=behind, drafts=drafts, strided=rng.random() < 0.4)
        elif op == "verify":
            c = dict(op=op, logits=rng.choice(["f32", "bf16", "f16"]), n=_log_uniform(rng, 1, 64), k=rng.choice([1, 2, 3, 4, 5, 7, 12]),
                     vocab=rng.choice([VOCAB, _log_uniform(rng, 40, 152000)]), drafter=rng.random() < 0.6, temperature=rng.choice([1.0, 0.6, 1.3, 0.0, -1.0]),
                     ragged=rng.random() < 0.4)
        else:
            n, longest = _log_uniform(rng, 1, 64), _log_uniform(rng, 1, 131072)
            lens = dict(shortest=rng.choice([longest, longest // 2, 1]), longest=longest)
            if op == "bound":
                c = dict(op=op, **shape, n_seqs=n, **lens, new=rng.choice([0, 1, 1, 5, 200]))
            else:
                keep = min(_log_uniform(rng, 3, 512), max(3, -(-longest // shape["page_tokens"])))
                c = dict(op=op, **shape, **queries, n_seqs=n, **lens, keep=keep)
                if op == "pick":
                    c.update(first=rng.choice([0, 1, 1, 2]), last=1)
        if _cost(c) <= most and _pool_bytes(c) < 6e8:
            return c


# ---- sizes ----------------------------------------------------------------------------------------------------

def _spread(lo, hi, n):
    """n whole numbers spread evenly between two bounds, the largest first."""
    return [hi - (hi - lo) * i // max(1, n - 1) for i in range(n)]


def _context(c):
    """(shared positions of each group, cached positions of each row) of a shared case."""
    shared = _spread(c["prefix_least"], c["prefix"], c["groups"])
    rows = c["groups"] * c["width"]
    if c["drafts"]:   # one sequence a group: its last `width` positions are the rows themselves
        return shared, [n - c["width"] + 1 + w for n in shared for w in range(c["width"])]
    behind = _spread(c["behind_least"], c["behind"], rows)
    return shared, [shared[r // c["width"]] + behind[r] for r in range(rows)]


def _blocks(c, n):
    return -(-n // c["page_tokens"])


def _n_pages(c):
    t = c["page_tokens"]
    if c["op"] == "shared":
        shared, lens = _context(c)
        if c["drafts"]:
            return max(1, sum(_blocks(c, n) for n in shared))
        # (a row's own pages begin with the one in which the shared positions end)
        return max(1, sum(n // t for n in shared) + sum(_blocks(c, n) - shared[r // c["width"]] // t for r, n in enumerate(lens)) + c["groups"])
    if c["op"] == "picked":  # (only the picked pages exist)
        return max(1, c["kv_heads"] * sum(min(c["keep"], _blocks(c, n)) for n in _spread(c["shortest"], c["longest"], c["n_seqs"])))
    return max(1, sum(_blocks(c, n) for n in _spread(c["shortest"], c["longest"], c["n_seqs"])))


def _k_row_bytes(c):
    return c["kv_heads"] * (c["head_dim"] * BYTES[c["store"]] + (4 if c["store"] in TOP else 0))


def _pool_bytes(c):
    if c["op"] == "verify":
        return 0
    if c["op"] == "pick":
        return 2 * _n_pages(c) * c["kv_heads"] * c["head_dim"] * BYTES[_bound_type(c["store"])]
    return 2 * _n_pages(c) * c["page_tokens"] * _k_row_bytes(c)


def _picked_lens(c, n):
    """Positions of the picked pages of a sequence of n: full ones and, last, the one in which the sequence ends."""
    t, blocks = c["page_tokens"], _blocks(c, n)
    return 0 if n == 0 else (min(c["keep"], blocks) - 1) * t + n - (blocks - 1) * t


def work(case):
    c = case
    if c["op"] == "verify":
        rows = c["n"] * (c["k"] + 1) + (c["n"] * c["k"] if c["drafter"] else 0)
        return {"bytes": rows * c["vocab"] * BYTES[c["logits"]] + 12 * c["n"] * (c["k"] + 1), "flops": 4 * rows * c["vocab"]}
    if c["op"] == "shared":
        shared, lens = _context(c)
        own_rows = 0 if c["drafts"] else sum(n - shared[r // c["width"]] for r, n in enumerate(lens))
        heads = c["kv_heads"] * c["group"]
        return {"bytes": 2 * (sum(shared) + own_rows) * _k_row_bytes(c) + 2 * len(lens) * heads * c["head_dim"] * BYTES[c["q"]],
                "flops": 4 * sum(lens) * heads * c["head_dim"]}
    lens = _spread(c["shortest"], c["longest"], c["n_seqs"])
    if c["op"] == "bound":
        t, rows, pages = c["page_tokens"], 0, 0
        for n in lens:
            first = (max(0, n - c["new"]) if c["new"] else 0) // t
            rows, pages = rows + max(0, n - first * t), pages + max(0, _blocks(c, n) - first)
        return {"bytes": rows * _k_row_bytes(c) + 2 * pages * c["kv_heads"] * c["head_dim"] * BYTES[_bound_type(c["store"])] + 4 * pages,
                "flops": 2 * rows * c["kv_heads"] * c["head_dim"]}
    q = c["n_seqs"] * c["kv_heads"] * c["group"] * c["head_dim"]
    if c["op"] == "pick":
        pages = _n_pages(c)
        return {"bytes": 2 * pages * c["kv_heads"] * c["head_dim"] * BYTES[_bound_type(c["store"])] + q * BYTES[c["q"]] + 4 * pages + 4 * c["n_seqs"] * c["kv_heads"] * c["keep"],
                "flops": 4 * pages * c["kv_heads"] * c["group"] * c["head_dim"]}
    seen = sum(_picked_lens(c, n) for n in lens)
    return {"bytes": 2 * seen * _k_row_bytes(c) + 2 * q * BYTES[c["q"]], "flops": 4 * seen * c["kv_heads"] * c["group"] * c["head_dim"]}


# ---- inputs ---------------------------------------------------------------------------------------------------

def _pool(c, gen):
    """A pool of values as a model leaves them: about unit variance, rows of different size."""
    shape = (1, _n_pages(c), c["kv_heads"], c["page_tokens"], c["head_dim"])
    parts, scales = [], []
    for _ in range(2):
        x = torch.randn(shape, generator=gen, device=DEVICE, dtype=torch.float32)
        if c["store"] in TOP:
            x.mul_(TOP[c["store"]] / 4).clamp_(-TOP[c["store"]], TOP[c["store"]])
            parts.append(x.round_().to(torch.int8) if c["store"] == "i8" else x.to(torch.float8_e4m3fn))
            scales.append((torch.rand(shape[:-1], generator=gen, device=DEVICE) + 0.5) * (4 / TOP[c["store"]]))
        else:
            parts.append(x.to(TORCH[c["store"]]))
            scales.append(None)
    return dict(k=parts[0], v=parts[1], k_scale=scales[0], v_scale=scales[1])


def _queries(c, gen, *rows):
    """Query rows, on request beside other heads, as in a fused projection."""
    heads = c["kv_heads"] * c["group"]
    wide = heads + 2 * c["kv_heads"] if c.get("strided") else heads
    return (torch.randn((*rows, wide, c["head_dim"]), generator=gen, device=DEVICE) * 1.5).to(TORCH[c["q"]])[..., :heads, :]


def _ints(x):
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.int32)).to(DEVICE)


def _inputs(case, seed):
    c = case
    gen = torch.Generator(device=DEVICE).manual_seed(seed)
    rng = np.random.default_rng(seed)
    if c["op"] == "verify":
        return _draft_inputs(c, gen, rng)
    if c["op"] == "shared":
        s = _pool(c, gen)
        shared, lens = _context(c)
        rows, width, t = len(lens), c["width"], c["page_tokens"]
        free = iter(rng.permutation(_n_pages(c)).tolist())   # pages in the order that a server's allocator leaves: scattered
        most = max(1, max(_blocks(c, n) for n in (shared if c["drafts"] else lens)))
        table = np.zeros((c["groups"] if c["drafts"] else rows, most), np.int32)
        for g, n in enumerate(shared):
            if c["drafts"]:
                table[g, :_blocks(c, n)] = [next(free) for _ in range(_blocks(c, n))]
                continue
            full = [next(free) for _ in range(n // t)]
            for r in range(g * width, (g + 1) * width):      # (the page that is not full is every row's own, with the same rows)
                mine = [next(free) for _ in range(_blocks(c, lens[r]) - n // t)]
                table[r, :len(full) + len(mine)] = full + mine
                if n % t and r > g * width:
                    for x in s.values():
                        if x is not None:
                            y = x.view(torch.uint8) if x.dtype == torch.float8_e4m3fn else x
                            y[0, mine[0], :, :n % t] = y[0, int(table[g * width, n // t]), :, :n % t]
        s.update(tables=_ints(table), lens=_ints(np.reshape(lens, (c["groups"], width))), prefix=_ints(shared), q=_queries(c, gen, c["groups"], width))
        return s
    lens = _spread(c["shortest"], c["longest"], c["n_seqs"])
    most = max(1, max(_blocks(c, n) for n in lens))
    if c["op"] == "picked":
        s = _pool(c, gen)
        n, hk = c["n_seqs"], c["kv_heads"]
        free, at = rng.permutation(_n_pages(c)), 0
        table, seen = np.full((n, hk, c["keep"]), -1, np.int32), np.zeros((n, hk), np.int32)
        for i, length in enumerate(lens):
            blocks = min(c["keep"], _blocks(c, length))
            table[i, :, :blocks] = free[at:at + hk * blocks].reshape(hk, blocks)
            seen[i], at = _picked_lens(c, length), at + hk * blocks
        s.update(tables=_ints(table), lens=_ints(seen), q=_queries(c, gen, n))
        return s
    free, at = rng.permutation(_n_pages(c)), 0
    table = np.zeros((c["n_seqs"], most), np.int32)
    for i, length in enumerate(lens):
        table[i, :_blocks(c, length)] = free[at:at + _blocks(c, length)]
        at += _blocks(c, length)
    shape = (1, _n_pages(c), c["kv_heads"], c["head_dim"])
    middle = torch.randn(shape, generator=gen, device=DEVICE) * 0.7
    half = torch.rand(shape, generator=gen, device=DEVICE) * 1.5 + 0.5
    s = dict(tables=_ints(table), lens=_ints(lens), lo=(middle - half).to(TORCH[_bound_type(c["store"])]), hi=(middle + half).to(TORCH[_bound_type(c["store"])]))
    if c["op"] == "bound":
        s.update(_pool(c, gen), since=_ints([max(0, n - c["new"]) if c["new"] else 0 for n in lens]))
    else:
        s.update(q=_queries(c, gen, c["n_seqs"]))
    return s


def _draft_inputs(c, gen, rng):
    """Logits of a model and of a cheaper one that is mostly of its opinion, and tokens drawn from the cheaper one."""
    n, k, v = c["n"], c["k"], c["vocab"]
    draft = (torch.randn((n, k, v), generator=gen, device=DEVICE) * 2.5).to(TORCH[c["logits"]])
    target = torch.randn((n, k + 1, v), generator=gen, device=DEVICE) * 0.5
    target[:, :k] += draft.float()
    target[:, k] *= 5
    target = target.to(TORCH[c["logits"]])
    s = dict(logits=target, uniforms=torch.rand((n, k + 1), generator=gen, device=DEVICE))
    t = torch.full((n,), c["temperature"], device=DEVICE)
    if c["temperature"] < 0:   # a server's mixture
        t = torch.tensor([0.0, 0.7, 1.0, 1.2], device=DEVICE)[torch.from_numpy(rng.integers(0, 4, n)).to(DEVICE)]
    warm = torch.where(t == 0, 1.0, t)[:, None, None]
    if c["drafter"]:
        noise = -torch.log(-torch.log(torch.rand((n, k, v), generator=gen, device=DEVICE).clamp(1e-7, 1 - 1e-7)))
        s["draft_logits"] = draft
        tokens = torch.where(t[:, None] == 0, draft.argmax(-1), (draft.float() / warm + noise).argmax(-1))
    else:
        s["draft_logits"] = None
        sure = torch.rand((n, k), generator=gen, device=DEVICE) < 0.7
        tokens = torch.where(sure, target[:, :k].argmax(-1), torch.from_numpy(rng.integers(0, v, (n, k))).to(DEVICE))
        if not t.any():
            tokens = target[:, :k].argmax(-1)
        elif n:   # (a draft that is found in the prompt is mostly what the model is sure of)
            target[:, :k].scatter_(2, tokens[..., None], (target[:, :k].float().amax(-1, keepdim=True) + 9).to(target.dtype))
    s["drafts"] = tokens.int()
    s["counts"] = _ints(rng.integers(0, k + 1, n)) if c["ragged"] else None
    s["temperature"] = t if c["temperature"] < 0 else c["temperature"]
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    if own:
        from paper_2512_21571_amd import binding
        s["binding"] = binding
        if case["op"] in ("shared", "picked", "bound"):
            s["pages"] = binding.Pages(s["k"], s["v"], s["k_scale"], s["v_scale"])
        elif case["op"] == "pick":   # (only the bounds are looked at; the pool is whatever the server has)
            c, t = case, TORCH[case["store"]]
            pool = [torch.zeros((1, _n_pages(c), c["kv_heads"], c["page_tokens"], c["head_dim"]), dtype=torch.uint8, device=DEVICE).to(t) for _ in range(2)]
            scales = [torch.ones(pool[0].shape[:-1], device=DEVICE) if c["store"] in TOP else None for _ in range(2)]
            s["pages"] = binding.Pages(*pool, *scales)
    return s


# ---- plain forms ----------------------------------------------------------------------------------------------

def _gather(pool, scales, page, row):
    """Rows [..., kv head, dim] of a layer's pages in fp32."""
    x = pool[0].view(torch.uint8)[page, :, row].view(pool.dtype).float() if pool.dtype == torch.float8_e4m3fn else pool[0][page, :, row].float()
    return x if scales is None else x * scales[0][page, :, row].unsqueeze(-1)


def _softmax_product(x, v):
    """exp(x) v / sum exp(x) over the last axis; rows of -infinity give zeros."""
    top = x.amax(-1, keepdim=True)
    e = torch.exp(x - torch.where(top == -math.inf, torch.zeros_like(top), top))
    total = e.sum(-1, keepdim=True)
    return torch.matmul(e, v) / torch.where(total == 0, torch.ones_like(total), total)


def _plain_shared(s):
    c, t = s["case"], s["case"]["page_tokens"]
    groups, width, hk, grp, d = c["groups"], c["width"], c["kv_heads"], c["group"], c["head_dim"]
    shared, lens = _context(c)
    out = []
    for g in range(groups):
        rows = [g] if c["drafts"] else list(range(g * width, (g + 1) * width))
        most = max(lens[g * width:(g + 1) * width])
        k, v, keep = [], [], []
        for i, r in enumerate(rows):     # the shared positions once, then those of every row; a row sees its own
            begin, end = (0 if i == 0 else shared[g]), (most if c["drafts"] else lens[r])
            p = torch.arange(begin, max(begin, end), device=DEVICE)
            page, at = s["tables"][r, p // t].long(), p % t
            k.append(_gather(s["k"], s["k_scale"], page, at))
            v.append(_gather(s["v"], s["v_scale"], page, at))
            w = torch.arange(width, device=DEVICE)[:, None]
            keep.append((p < s["lens"][g].long()[:, None]) & ((p < s["prefix"][g]) | (w == i) | c["drafts"]))
        k, v, keep = torch.cat(k).permute(1, 2, 0).contiguous(), torch.cat(v).permute(1, 0, 2).contiguous(), torch.cat(keep, 1)
        q = s["q"][g].float().reshape(width, hk, grp, d).transpose(0, 1).reshape(hk, width * grp, d) / math.sqrt(d)
        x = torch.matmul(q, k).reshape(hk, width, grp, -1).masked_fill(~keep[:, None], -math.inf).reshape(hk, width * grp, -1)
        o = _softmax_product(x, v) if x.shape[-1] else torch.zeros_like(q)
        out.append(o.reshape(hk, width, grp, d).transpose(0, 1).reshape(width, hk * grp, d))
    return torch.stack(out).to(s["q"].dtype)


def _plain_picked(s):
    c, t = s["case"], s["case"]["page_tokens"]
    n, hk, grp, d = c["n_seqs"], c["kv_heads"], c["group"], c["head_dim"]
    p = torch.arange(c["keep"] * t, device=DEVICE)
    page, row = s["tables"][:, :, p // t].long().clamp(min=0), (p % t)
    head = torch.arange(hk, device=DEVICE)[:, None]

    def rows(pool, scales):
        x = pool[0].view(torch.uint8)[page, head, row].view(pool.dtype).float() if pool.dtype == torch.float8_e4m3fn else pool[0][page, head, row].float()
        return x if scales is None else x * scales[0][page, head, row].unsqueeze(-1)

    q = s["q"].float().reshape(n, hk, grp, d) / math.sqrt(d)
    x = torch.matmul(q, rows(s["k"], s["k_scale"]).transpose(2, 3).contiguous())
    x = x.masked_fill((p >= s["lens"].long()[..., None])[:, :, None], -math.inf)
    return _softmax_product(x, rows(s["v"], s["v_scale"])).reshape(n, hk * grp, d).to(s["q"].dtype)


def _plain_verify(s):
    """In 64 bits: a running sum over a whole vocabulary is compared with a random number."""
    c = s["case"]
    n, k, v = c["n"], c["k"], c["vocab"]
    t = s["temperature"] if isinstance(s["temperature"], torch.Tensor) else torch.full((n,), s["temperature"], device=DEVICE)

    def probabilities(x):
        x = x.double()
        warm = torch.where(t == 0, torch.ones_like(t), t).double()[:, None, None]
        top = x.amax(-1, keepdim=True)
        e = torch.exp((x - top) / warm)
        index = torch.arange(v, device=DEVICE)
        best = torch.where(x == top, index, v).amin(-1, keepdim=True)       # greedy: the lowest index of the largest
        return torch.where((t == 0)[:, None, None], (index == best).double(), e / e.sum(-1, keepdim=True))

    p = probabilities(s["logits"])
    at = s["drafts"].long()[..., None]
    if s["draft_logits"] is not None:
        q = probabilities(s["draft_logits"])
    else:
        q = torch.zeros_like(p[:, :k]).scatter_(2, at, 1.0)
    count = torch.full((n,), k, device=DEVICE) if s["counts"] is None else s["counts"].long()
    u = s["uniforms"].double()
    fine = (u[:, :k] * q.gather(2, at)[..., 0] < p[:, :k].gather(2, at)[..., 0]) & (torch.arange(k, device=DEVICE) < count[:, None])
    accepted = torch.cumprod(fine.long(), 1).sum(1)
    i = torch.arange(n, device=DEVICE)
    full = p[i, accepted]
    rest = torch.clamp(full - q[i, accepted.clamp(max=k - 1)], min=0)
    rest = torch.where(((accepted == count) | (rest.sum(-1) == 0))[:, None], full, rest)
    sums = torch.cumsum(rest, -1)
    token = (sums <= u[:, k:] * sums[:, -1:]).sum(-1)
    j = torch.arange(k + 1, device=DEVICE)
    tokens = torch.where(j < accepted[:, None], torch.cat([s["drafts"].long(), token[:, None]], 1), torch.where(j == accepted[:, None], token[:, None], -1))
    return [tokens.int(), accepted.int()]


def _outwards(x, up):
    """float64 -> the nearest bf16 that is not below (above) it."""
    y = x.float().to(torch.bfloat16)
    wrong = (y.double() < x) if up else (y.double() > x)
    bits = y.view(torch.int16).int() & 0xffff
    away = (y > 0) if up else (y < 0)             # to a larger magnitude, else to a smaller one; zero to the least number of that sign
    bits = torch.where((y == 0), torch.full_like(bits, 1 if up else 0x8001), torch.where(away, bits + 1, bits - 1))
    return torch.where(wrong, (bits - ((bits & 0x8000) << 1)).short().view(torch.bfloat16), y)


def _plain_bound(s):
    c, t = s["case"], s["case"]["page_tokens"]
    n, most = s["tables"].shape
    block = torch.arange(most, device=DEVICE)
    first = (s["since"].long() // t)[:, None]
    seq, block = torch.nonzero((block >= first) & (block * t < s["lens"].long()[:, None]), as_tuple=True)
    page = s["tables"][seq, block].long()
    x = (s["k"][0].view(torch.uint8)[page].view(s["k"].dtype) if s["k"].dtype == torch.float8_e4m3fn else s["k"][0][page])   # [page, head, row, dim]
    x = x.float() if s["k_scale"] is None else x.float().double() * s["k_scale"][0][page].double()[..., None]
    there = (torch.arange(t, device=DEVICE) < (s["lens"].long()[seq] - block * t)[:, None])[:, None, :, None]
    lo, hi = torch.where(there, x, math.inf).amin(2), torch.where(there, x, -math.inf).amax(2)
    s["lo"][0, page] = _outwards(lo, False) if c["store"] in TOP else lo.to(s["lo"].dtype)
    s["hi"][0, page] = _outwards(hi, True) if c["store"] in TOP else hi.to(s["hi"].dtype)
    return [s["lo"], s["hi"]]


def _plain_pick(s):
    """In 64 bits: the scores of two pages may be close."""
    c, t = s["case"], s["case"]["page_tokens"]
    n, hk, grp, d, keep = c["n_seqs"], c["kv_heads"], c["group"], c["head_dim"], c["keep"]
    most = s["tables"].shape[1]
    q = s["q"].double().reshape(n, hk, grp, d)
    lo, hi = (s[b][0][s["tables"].long()].double().permute(0, 2, 3, 1).contiguous() for b in ("lo", "hi"))      # [n, kv head, dim, block]
    score = (torch.matmul(q.clamp(min=0), hi) + torch.matmul(q.clamp(max=0), lo)).amax(2)
    block = torch.arange(max(most, keep), device=DEVICE)
    blocks = -(-s["lens"].long() // t)[:, None, None]
    score = torch.cat([score, score.new_full((n, hk, max(0, keep - most)), -math.inf)], 2)
    score = torch.where((block < c["first"]) | (block >= blocks - c["last"]), math.inf, score)
    score = torch.where(block < blocks, score, -math.inf)
    best = torch.argsort(score, dim=2, descending=True, stable=True)[..., :keep]
    best = torch.where(best < blocks, best, len(block)).sort(-1)[0]                                            # in order; what is not there last
    tables = torch.cat([s["tables"], s["tables"].new_full((n, len(block) + 1 - most), -1)], 1)[:, None].expand(n, hk, -1)
    lens = s["lens"].long()[:, None].expand(n, hk)
    count = blocks[..., 0].clamp(max=keep)
    return [tables.gather(2, best), torch.where(lens > 0, (count - 1) * t + lens - (blocks[..., 0] - 1) * t, 0).int()]


# ---- one pass --------------------------------------------------------------------------------------------------

def run(state):
    s, c = state, state["case"]
    op = c["op"]
    if not own:
        return {"shared": _plain_shared, "verify": _plain_verify, "bound": _plain_bound, "pick": _plain_pick, "picked": _plain_picked}[op](s)
    if op == "shared":
        if c["drafts"]:
            return s["pages"].attention_shared(0, s["q"], s["tables"], s["lens"], max_len=c["prefix"])
        return s["pages"].attention_shared(0, s["q"], s["tables"], s["lens"], s["prefix"], max_len=c["prefix"] + c["behind"], max_own=c["behind"])
    if op == "verify":
        return list(s["binding"].draft_verify(s["logits"], s["drafts"], s["uniforms"], s["draft_logits"], counts=s["counts"], temperature=s["temperature"]))
    if op == "bound":
        s["pages"].bound(0, (s["lo"], s["hi"]), s["tables"], s["lens"], since=s["since"], max_new=c["new"])
        return [s["lo"], s["hi"]]
    if op == "pick":
        return list(s["pages"].pick(0, (s["lo"], s["hi"]), s["q"], s["tables"], s["lens"], c["keep"], first=c["first"], last=c["last"]))
    return s["pages"].attention(0, s["q"], s["tables"], s["lens"])


# ---- the definition in 64 bits ----------------------------------------------------------------------------------

def _values(pool, scales, page, head):
    """Pages of one head as float64 [pages * rows, dim]."""
    x = pool.view(torch.uint8)[0, page, head].view(pool.dtype) if pool.dtype == torch.float8_e4m3fn else pool[0, page, head]
    x = x.to(torch.float32).double()
    x = x if scales is None else x * scales[0, page, head].double()[..., None]
    return x.reshape(-1, x.shape[-1])


def _row_softmax(s, q, page, head, n):
    k, v = (_values(s[a], s[a + "_scale"], page, head)[:n] for a in ("k", "v"))
    return torch.softmax((q.double() @ k.T) * q.shape[-1] ** -0.5, -1) @ v if n else torch.zeros_like(q, dtype=torch.float64)


def exact(case, seed):
    c, s = case, _inputs(case, seed)
    t = c.get("page_tokens", 1)
    if c["op"] == "shared":
        lens, width, grp = _context(c)[1], c["width"], c["group"]
        out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEVICE)
        for r, n in enumerate(lens):     # every row by itself, through its own table
            page = s["tables"][r // width if c["drafts"] else r, :-(-n // t)].long()
            for h in range(c["kv_heads"]):
                out[r // width, r % width, h * grp:(h + 1) * grp] = _row_softmax(s, s["q"][r // width, r % width, h * grp:(h + 1) * grp], page, h, n)
        return out
    if c["op"] == "picked":
        grp = c["group"]
        out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEVICE)
        for i, length in enumerate(_spread(c["shortest"], c["longest"], c["n_seqs"])):
            n = _picked_lens(c, length)
            for h in range(c["kv_heads"]):
                out[i, h * grp:(h + 1) * grp] = _row_softmax(s, s["q"][i, h * grp:(h + 1) * grp], s["tables"][i, h, :-(-n // t)].long(), h, n)
        return out
    if c["op"] == "verify":
        n, k = c["n"], c["k"]
        tokens, accepted = np.full((n, k + 1), -1, np.int32), np.zeros(n, np.int32)
        u, drafts = s["uniforms"].double().cpu().numpy(), s["drafts"].cpu().numpy()
        heat = s["temperature"].cpu().numpy() if isinstance(s["temperature"], torch.Tensor) else np.full(n, s["temperature"], np.float32)

        def distribution(x, i):
            x = x.double().cpu().numpy()
            if heat[i] == 0:
                return (np.arange(len(x)) == int(np.argmax(x))).astype(np.float64)
            e = np.exp((x - x.max()) / float(heat[i]))
            return e / e.sum()

        for i in range(n):
            count = k if s["counts"] is None else int(s["counts"][i])
            j = 0
            while True:
                r = p = distribution(s["logits"][i, j], i)
                if j == count:
                    break
                x = drafts[i, j]
                q = distribution(s["draft_logits"][i, j], i) if c["drafter"] else (np.arange(c["vocab"]) == x).astype(np.float64)
                if not u[i, j] * q[x] < p[x]:
                    r = np.maximum(p - q, 0)
                    r = r if r.sum() > 0 else p
                    break
                tokens[i, j], j = x, j + 1
            sums = np.cumsum(r)
            tokens[i, j], accepted[i] = int(np.searchsorted(sums, u[i, k] * sums[-1], side="right")), j
        return [torch.from_numpy(tokens), torch.from_numpy(accepted)]
    tables, lens = s["tables"].cpu().numpy(), _spread(c["shortest"], c["longest"], c["n_seqs"])
    if c["op"] == "bound":
        lo, hi = s["lo"].double(), s["hi"].double()
        for i, n in enumerate(lens):
            for b in range((max(0, n - c["new"]) if c["new"] else 0) // t, -(-n // t)):
                page, rows = int(tables[i, b]), min(t, n - b * t)
                x = (s["k"].view(torch.uint8)[0, page].view(s["k"].dtype) if s["k"].dtype == torch.float8_e4m3fn else s["k"][0, page])[:, :rows].float().double()
                x = x if s["k_scale"] is None else x * s["k_scale"][0, page, :, :rows].double()[..., None]
                lo[0, page], hi[0, page] = x.amin(1), x.amax(1)
                if c["store"] in TOP:   # steps of bf16: 2^-7 of the power of two below
                    for y, rounded in ((lo, torch.floor), (hi, torch.ceil)):
                        step = torch.ldexp(torch.ones_like(y[0, page]), torch.frexp(y[0, page])[1] - 8)
                        y[0, page] = rounded(y[0, page] / step) * step
        return [lo, hi]
    grp, hk, keep = c["group"], c["kv_heads"], c["keep"]
    picked, seen = np.full((c["n_seqs"], hk, keep), -1, np.int32), np.zeros((c["n_seqs"], hk), np.int32)
    q = s["q"].double()
    for i, n in enumerate(lens):
        blocks = -(-n // t)
        page = s["tables"][i, :blocks].long()
        for h in range(hk):
            lo, hi = s["lo"][0, page, h].double(), s["hi"][0, page, h].double()
            score = torch.stack([torch.maximum(x * lo, x * hi).sum(-1) for x in q[i, h * grp:(h + 1) * grp]]).amax(0).cpu().numpy()
            always = {b for b in range(blocks) if b < c["first"] or b >= blocks - c["last"]}
            order = sorted(always) + [int(b) for b in np.argsort(-score, kind="stable") if int(b) not in always]
            chosen = sorted(order[:keep])
            picked[i, h, :len(chosen)] = tables[i, chosen]
            seen[i, h] = (len(chosen) - 1) * t + n - (blocks - 1) * t if n else 0
    return [torch.from_numpy(picked), torch.from_numpy(seen)]
