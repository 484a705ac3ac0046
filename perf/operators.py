"""Timed operators of a paged KV cache: what a server that keeps many sequences, or the hypotheses of a beam
search, in pages of a few bits has the library do next to a model's matrix products.

* ``append``   rows of K and V go into the pages that a table names, 8-bit caches quantised as they are written
* ``read``     positions of the cache come back as rows
* ``attention`` one new token of every sequence against its cached positions
* ``select``   the best continuations of every beam of a search, out of beams x vocabulary
* ``reorder``  the beams take over the pages of the beams that they continue

A pool of pages is ``k, v [layer][page][kv head][row of the page][head_dim]``; 8-bit pools have one fp32 scale
for each row of 128 (or 64) values in ``k_scale, v_scale [layer][page][kv head][row of the page]``.  A table gives
for every sequence the pages of its positions in order: position p is row p % page_tokens of entry p // page_tokens.

Shapes are those of the repository's own models (0.6B: 16 query and 8 kv heads, 4B and 8B: 32 and 8, heads of
128, a vocabulary of 151936) and generic ones around them.
"""
import math

import numpy as np
import torch

own = False

DEVICE = "cuda:0"
TORCH = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16, "i8": torch.int8, "e4m3": torch.float8_e4m3fn}
BYTES = {"f32": 4, "bf16": 2, "f16": 2, "i8": 1, "e4m3": 1}
TOP = {"i8": 127.0, "e4m3": 448.0}     # largest magnitude that a stored value stands for, before its scale
LEAST_SCALE = 2.0 ** -80               # scales are not smaller: a row of zeros has this one
VOCAB = 151936


def listed():
    return [
        # one decode step of sixteen sequences: their new rows, as the projection leaves them (launch latency)
        dict(name="append-i8-b16", op="append", store="i8", rows="f32", n_rows=16, n_seqs=16, kv_heads=8, head_dim=128, page_tokens=16, ctx=4096, strided=True),
        # a full prompt block moves into pages
        dict(name="append-e4m3-p4096", op="append", store="e4m3", rows="bf16", n_rows=4096, n_seqs=1, kv_heads=8, head_dim=128, page_tokens=64, ctx=4096, strided=False),
        # a cached document comes back for a second use
        dict(name="read-i8-p4096", op="read", store="i8", rows="bf16", n_rows=4096, n_seqs=1, kv_heads=8, head_dim=128, page_tokens=16, ctx=4096, strided=False),
        # odd numbers of rows of a few sequences, inspected in fp32
        dict(name="read-e4m3-ragged", op="read", store="e4m3", rows="f32", n_rows=333, n_seqs=3, kv_heads=5, head_dim=64, page_tokens=24, ctx=500, strided=False),
        # one user of the smallest model early in a chat
        dict(name="attn-bf16-b1-c100", op="attention", store="bf16", q="bf16", n_seqs=1, kv_heads=8, group=2, head_dim=128, page_tokens=16, longest=100, shortest=100, window=0),
        # the largest configuration: sixteen full contexts, queries as the projection leaves them
        dict(name="attn-bf16-b16-c4096", op="attention", store="bf16", q="f32", n_seqs=16, kv_heads=8, group=4, head_dim=128, page_tokens=64, longest=4096, shortest=4096, window=0),
        # a server's batch of contexts of different lengths in an 8-bit cache
        dict(name="attn-i8-b48-ragged", op="attention", store="i8", q="bf16", n_seqs=48, kv_heads=8, group=4, head_dim=128, page_tokens=16, longest=6000, shortest=1, window=0),
        # one user on a book: few rows, a long axis
        dict(name="attn-e4m3-b1-c131072", op="attention", store="e4m3", q="f16", n_seqs=1, kv_heads=8, group=4, head_dim=128, page_tokens=128, longest=131072, shortest=131072, window=0),
        # one search of four beams
        dict(name="select-g1-w4", op="select", logits="f32", groups=1, width=4, vocab=VOCAB, finished=0.0, masked=0.0),
        # a server's searches, some hypotheses ended, some tokens forbidden
        dict(name="select-g16-w8", op="select", logits="bf16", groups=16, width=8, vocab=VOCAB, finished=0.2, masked=0.01),
        # four beams of the 8B shape after a step, the last page not full
        dict(name="reorder-g1-w4", op="reorder", store="bf16", groups=1, width=4, layers=36, kv_heads=8, head_dim=128, page_tokens=16, ctx=523),
        # two searches of eight beams in an 8-bit cache of larger pages
        dict(name="reorder-i8-g2-w8", op="reorder", store="i8", groups=2, width=8, layers=28, kv_heads=8, head_dim=128, page_tokens=32, ctx=250),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _cost(case):
    w = work(case)
    return w["bytes"] / 6e12 + w["flops"] / 5e14


def draw(rng):
    most = max(_cost(c) for c in listed())
    while True:
        op = rng.choice(["append", "read", "attention", "attention", "attention", "select", "select", "reorder"])
        store = rng.choice(["bf16", "f16", "i8", "e4m3", "i8", "e4m3", "f32"])
        heads, dim, page = rng.choice([1, 2, 3, 4, 5, 8, 8, 16]), rng.choice([64, 128, 128]), rng.choice([8, 16, 16, 24, 32, 64, 128])
        if op in ("append", "read"):
            n_seqs = rng.choice([1, 1, 2, 7, 16, 40])
            n_rows = max(n_seqs, _log_uniform(rng, 1, 8192))
            c = dict(op=op, store=store, rows=rng.choice(["f32", "bf16", "f16"]), n_rows=n_rows, n_seqs=n_seqs, kv_heads=heads, head_dim=dim,
                     page_tokens=page, ctx=-(-n_rows // n_seqs) + rng.randint(0, 300), strided=op == "append" and rng.random() < 0.5)
        elif op == "attention":
            n_seqs = _log_uniform(rng, 1, 64)
            longest = _log_uniform(rng, 1, 131072)
            c = dict(op=op, store=store, q=rng.choice(["f32", "bf16", "f16"]), n_seqs=n_seqs, kv_heads=heads, group=rng.choice([1, 2, 3, 4, 5, 8, 16]), head_dim=dim,
                     page_tokens=page, longest=longest, shortest=rng.choice([longest, longest // 2, 0]), window=rng.choice([0, 0, 0, _log_uniform(rng, 1, 4096)]))
        elif op == "select":
            c = dict(op=op, logits=rng.choice(["f32", "bf16", "f16"]), groups=_log_uniform(rng, 1, 24), width=rng.choice([1, 2, 3, 4, 5, 8, 12, 16]),
                     vocab=rng.choice([VOCAB, _log_uniform(rng, 40, 152000)]), finished=rng.choice([0.0, 0.3]), masked=rng.choice([0.0, 0.02, 0.6]))
        else:
            c = dict(op=op, store=store, groups=rng.choice([1, 1, 2, 4]), width=rng.choice([2, 3, 4, 5, 8, 16]), layers=rng.randint(1, 36), kv_heads=heads,
                     head_dim=dim, page_tokens=page, ctx=_log_uniform(rng, 1, 700))
        if _cost(c) <= most and _pool_bytes(c) < 6e8:
            return c


# ---- sizes ----------------------------------------------------------------------------------------------------

def _lens(c):
    """Cached positions of each sequence of an attention case: spread evenly between the two bounds, the longest first."""
    n = c["n_seqs"]
    return [c["longest"] - (c["longest"] - c["shortest"]) * i // max(1, n - 1) for i in range(n)]


def _n_pages(c):
    t = c["page_tokens"]
    if c["op"] == "attention":
        return max(1, sum(-(-n // t) for n in _lens(c)))
    if c["op"] == "reorder":  # every group's full pages, two pages of its own for every beam (before and after)
        return c["groups"] * (c["ctx"] // t + 2 * c["width"])
    return c["n_seqs"] * -(-c["ctx"] // t)


def _row_bytes(c):
    return c["kv_heads"] * (c["head_dim"] * BYTES[c["store"]] + (4 if c["store"] in TOP else 0))


def _pool_bytes(c):
    if c["op"] == "select":
        return 0
    return 2 * c.get("layers", 1) * _n_pages(c) * c["page_tokens"] * _row_bytes(c)


def work(case):
    c = case
    if c["op"] in ("append", "read"):
        rows = 2 * c["n_rows"] * (c["kv_heads"] * c["head_dim"] * BYTES[c["rows"]] + _row_bytes(c))
        return {"bytes": rows + 12 * c["n_rows"], "flops": 4 * c["n_rows"] * c["kv_heads"] * c["head_dim"]}
    if c["op"] == "attention":
        seen = sum(min(n, c["window"]) if c["window"] else n for n in _lens(c))
        q = c["n_seqs"] * c["kv_heads"] * c["group"] * c["head_dim"]
        return {"bytes": 2 * seen * _row_bytes(c) + 2 * q * BYTES[c["q"]] + 4 * (_n_pages(c) + c["n_seqs"]),
                "flops": 4 * seen * c["kv_heads"] * c["group"] * c["head_dim"]}
    if c["op"] == "select":
        n = c["groups"] * c["width"]
        return {"bytes": n * (c["vocab"] * BYTES[c["logits"]] + 22), "flops": 4 * n * c["vocab"]}
    beams, full, part = c["groups"] * c["width"], c["ctx"] // c["page_tokens"], c["ctx"] % c["page_tokens"]
    return {"bytes": 4 * beams * (2 * full + 3) + 4 * beams * c["layers"] * part * _row_bytes(c), "flops": 0}


# ---- inputs ---------------------------------------------------------------------------------------------------

def _pool(c, gen):
    """A pool of values as a model leaves them: about unit variance, rows of different size."""
    shape = (c.get("layers", 1), _n_pages(c), c["kv_heads"], c["page_tokens"], c["head_dim"])
    scales, parts = [], []
    for _ in range(2):
        if c["store"] in TOP:
            x = torch.randn(shape, generator=gen, device=DEVICE, dtype=torch.float32).mul_(TOP[c["store"]] / 4).clamp_(-TOP[c["store"]], TOP[c["store"]])
            parts.append(x.round_().to(torch.int8) if c["store"] == "i8" else x.to(torch.float8_e4m3fn))
            scales.append((torch.rand(shape[:-1], generator=gen, device=DEVICE) + 0.5) * (4 / TOP[c["store"]]))
        else:
            parts.append(torch.randn(shape, generator=gen, device=DEVICE, dtype=torch.float32).to(TORCH[c["store"]]))
            scales.append(None)
    return parts[0], parts[1], scales[0], scales[1]


def _tables(c, rng, n_pages):
    """Pages in the order that a server's allocator leaves: scattered."""
    t = c["page_tokens"]
    per = [-(-n // t) for n in _lens(c)] if c["op"] == "attention" else [-(-c["ctx"] // t)] * c["n_seqs"]
    free = rng.permutation(n_pages)
    table, at = np.zeros((c["n_seqs"], max(1, max(per))), np.int32), 0
    for i, n in enumerate(per):
        table[i, :n] = free[at:at + n]
        at += n
    return torch.from_numpy(table).to(DEVICE)


def _inputs(case, seed):
    c = case
    gen = torch.Generator(device=DEVICE).manual_seed(seed)
    rng = np.random.default_rng(seed)
    s = {}
    if c["op"] == "select":
        g, w, v = c["groups"], c["width"], c["vocab"]
        x = torch.randn((g, w, v), generator=gen, device=DEVICE) * 2.5
        if c["masked"]:
            x.masked_fill_(torch.rand((g, w, v), generator=gen, device=DEVICE) < c["masked"], -math.inf)
        s["logits"] = x.to(TORCH[c["logits"]])
        s["scores"] = -(torch.rand((g, w), generator=gen, device=DEVICE) * 4 + 20)
        s["finished"] = torch.rand((g, w), generator=gen, device=DEVICE) < c["finished"]
        s["eos"] = int(rng.integers(0, v))
        return s
    s["k"], s["v"], s["k_scale"], s["v_scale"] = _pool(c, gen)
    if c["op"] in ("append", "read"):
        n, per = c["n_rows"], -(-c["n_rows"] // c["n_seqs"])
        s["tables"] = _tables(c, rng, _n_pages(c))
        # the last rows of each sequence: the i-th sequence has rows i * per .. of the n
        start = c["ctx"] - per
        i = np.arange(n)
        s["seq"] = torch.from_numpy((i // per).astype(np.int32)).to(DEVICE)
        s["pos"] = torch.from_numpy((start + i % per).astype(np.int32)).to(DEVICE)
        if c["op"] == "append":
            heads = (3 if c["strided"] else 1) * c["kv_heads"]  # (strided: K and V stand beside other heads, as in a fused projection)
            loud = torch.rand((n, heads, 1), generator=gen, device=DEVICE) * 2 + 0.25
            for name in ("k_rows", "v_rows"):
                x = (torch.randn((n, heads, c["head_dim"]), generator=gen, device=DEVICE) * loud).to(TORCH[c["rows"]])
                s[name] = x[:, heads - c["kv_heads"]:]
        return s
    if c["op"] == "attention":
        s["tables"] = _tables(c, rng, _n_pages(c))
        s["lens"] = torch.tensor(_lens(c), dtype=torch.int32, device=DEVICE)
        s["q"] = (torch.randn((c["n_seqs"], c["kv_heads"] * c["group"], c["head_dim"]), generator=gen, device=DEVICE) * 1.5).to(TORCH[c["q"]])
        return s
    g, w, full = c["groups"], c["width"], c["ctx"] // c["page_tokens"]
    pages = rng.permutation(_n_pages(c)).astype(np.int32).reshape(g, full + 2 * w)
    before, after = np.zeros((g, w, full + 1), np.int32), np.zeros((g, w, full + 1), np.int32)
    before[:, :, :full] = pages[:, None, :full]
    before[:, :, full], after[:, :, full] = pages[:, full:full + w], pages[:, full + w:]
    s["before"], s["after"] = (torch.from_numpy(t.reshape(g * w, full + 1)).to(DEVICE) for t in (before, after))
    s["lens"] = torch.full((g * w,), c["ctx"], dtype=torch.int32, device=DEVICE)
    s["parents"] = torch.from_numpy(rng.integers(0, w, (g, w)).astype(np.int32)).to(DEVICE)
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    if own:
        from paper_2512_21571_amd import binding
        s["binding"] = binding
        if case["op"] != "select":
            s["pages"] = binding.Pages(s["k"], s["v"], s["k_scale"], s["v_scale"])
    return s


# ---- plain forms ----------------------------------------------------------------------------------------------

def _to_e4m3(y):
    """float64 -> the nearest e4m3 value (ties to even), |y| at most 448 and a little."""
    _, e = torch.frexp(y)
    step = torch.ldexp(torch.ones_like(y), (e - 1).clamp(min=-6) - 3)
    return ((y / step).round() * step).clamp(-448, 448)


def _quantise(x, store):
    """Rows of any type -> (stored values, scales): scale = largest magnitude / TOP in fp32, value = x / scale rounded
    to the nearest.  In 64 bits: a value beside a border is one step off otherwise."""
    top = x.double().abs().amax(-1)
    scale = (top / torch.full_like(top, TOP[store])).float().clamp(min=LEAST_SCALE)
    y = x.double() / scale.double().unsqueeze(-1)
    return (y.round().to(torch.int8) if store == "i8" else _to_e4m3(y).float().to(torch.float8_e4m3fn)), scale


def _plain_append(s):
    c, t = s["case"], s["case"]["page_tokens"]
    page, row = s["tables"][s["seq"].long(), (s["pos"] // t).long()].long(), (s["pos"] % t).long()
    out = []
    for pool, scales, rows in ((s["k"], s["k_scale"], s["k_rows"]), (s["v"], s["v_scale"], s["v_rows"])):
        if c["store"] in TOP:
            val, sc = _quantise(rows, c["store"])
            pool[0].view(torch.uint8)[page, :, row] = val.view(torch.uint8)
            scales[0][page, :, row] = sc
            out += [pool, scales]
        else:
            pool[0][page, :, row] = rows.to(pool.dtype)
            out.append(pool)
    return out


def _gather(pool, scales, page, row):
    """Rows [..., kv head, dim] of a layer's pages in fp32."""
    x = pool[0].view(torch.uint8)[page, :, row].view(pool.dtype).float() if pool.dtype == torch.float8_e4m3fn else pool[0][page, :, row].float()
    return x if scales is None else x * scales[0][page, :, row].unsqueeze(-1)


def _plain_read(s):
    c, t = s["case"], s["case"]["page_tokens"]
    page, row = s["tables"][s["seq"].long(), (s["pos"] // t).long()].long(), (s["pos"] % t).long()
    return [_gather(pool, sc, page, row).to(TORCH[c["rows"]]) for pool, sc in ((s["k"], s["k_scale"]), (s["v"], s["v_scale"]))]


def _plain_attention(s):
    c, t = s["case"], s["case"]["page_tokens"]
    n, hk, g, d, longest = c["n_seqs"], c["kv_heads"], c["group"], c["head_dim"], c["longest"]
    if longest == 0:
        return torch.zeros_like(s["q"])
    p = torch.arange(longest, device=DEVICE)
    page, row = s["tables"][:, p // t].long(), (p % t).expand(n, -1)      # [n, longest]
    k = _gather(s["k"], s["k_scale"], page, row).permute(0, 2, 3, 1).contiguous()  # [n, kv head, dim, position]
    q = s["q"].float().reshape(n, hk, g, d) / math.sqrt(d)
    x = torch.matmul(q, k)
    lens = s["lens"].long()[:, None]
    keep = p[None] < lens
    if c["window"]:
        keep = keep & (p[None] >= lens - c["window"])
    x = x.masked_fill(~keep[:, None, None], -math.inf)
    top = x.amax(-1, keepdim=True)
    e = torch.exp(x - torch.where(top == -math.inf, torch.zeros_like(top), top))
    total = e.sum(-1, keepdim=True)
    v = _gather(s["v"], s["v_scale"], page, row).permute(0, 2, 1, 3).contiguous()
    out = torch.matmul(e, v) / torch.where(total == 0, torch.ones_like(total), total)
    return out.reshape(n, hk * g, d).to(s["q"].dtype)


def _plain_select(s):
    c = s["case"]
    g, w, v = c["groups"], c["width"], c["vocab"]
    x = s["logits"].double()                                              # scores of two beams may be close: 64 bits
    top = x.amax(-1, keepdim=True)
    lse = top + torch.log(torch.exp(x - top).sum(-1, keepdim=True))
    total = s["scores"].double().unsqueeze(-1) + torch.where(x == -math.inf, x, x - lse)
    least = torch.finfo(torch.float64).min
    total = torch.where(total == -math.inf, torch.full_like(total, least), total)  # forbidden, but there: below it, what is not there
    token = torch.arange(v, device=DEVICE)
    ended = s["finished"].unsqueeze(-1)
    total = torch.where(ended, torch.where(token == s["eos"], s["scores"].double().unsqueeze(-1), torch.full_like(total, -math.inf)), total)
    total = total.reshape(g, w * v)
    index = torch.arange(w * v, device=DEVICE)
    picked, values = [], []
    for _ in range(w):
        best = total.amax(-1, keepdim=True)
        at = torch.where(total == best, index, torch.full_like(index, w * v)).amin(-1, keepdim=True)   # ties: the lowest index
        picked.append(at)
        values.append(best)
        total = total.scatter(1, at, -math.inf)
    at, best = torch.cat(picked, 1), torch.cat(values, 1)
    best = torch.where(best == least, torch.full_like(best, -math.inf), best)
    tokens, parents = (at % v).int(), (at // v).int()
    ended = s["finished"].gather(1, parents.long()) | (tokens == s["eos"])
    return [tokens, parents, best.float(), ended]


def _plain_reorder(s):
    c = s["case"]
    g, w, t = c["groups"], c["width"], c["page_tokens"]
    full, part = c["ctx"] // t, c["ctx"] % t
    parent = (torch.arange(g, device=DEVICE)[:, None] * w + s["parents"].long()).reshape(-1)
    src, dst = s["before"][parent], s["after"]
    dst[:, :full] = src[:, :full]
    out = [dst]
    for pool, scales in ((s["k"], s["k_scale"]), (s["v"], s["v_scale"])):
        for x in (pool, scales):
            if x is None:
                continue
            if part:
                b = x.view(torch.uint8) if x.dtype == torch.float8_e4m3fn else x
                b[:, dst[:, full].long(), :, :part] = b[:, src[:, full].long(), :, :part]
            out.append(x)
    return out


# ---- one pass --------------------------------------------------------------------------------------------------

def run(state):
    s, op = state, state["case"]["op"]
    if not own:
        return {"append": _plain_append, "read": _plain_read, "attention": _plain_attention, "select": _plain_select, "reorder": _plain_reorder}[op](s)
    if op == "append":
        s["pages"].append(0, s["k_rows"], s["v_rows"], s["tables"], s["seq"], s["pos"])
        return [x for x in (s["k"], s["k_scale"], s["v"], s["v_scale"]) if x is not None]
    if op == "read":
        return list(s["pages"].read(0, s["tables"], s["seq"], s["pos"], dtype=TORCH[s["case"]["rows"]]))
    if op == "attention":
        return s["pages"].attention(0, s["q"], s["tables"], s["lens"], max_len=s["case"]["longest"], window=s["case"]["window"])
    if op == "select":
        return list(s["binding"].beam_select(s["logits"], s["scores"], s["finished"], eos=s["eos"]))
    s["pages"].reorder(s["before"], s["after"], s["lens"], s["parents"])
    return [s["after"]] + [x for x in (s["k"], s["k_scale"], s["v"], s["v_scale"]) if x is not None]


# ---- the definition in 64 bits ----------------------------------------------------------------------------------

_E4M3 = None


def _nearest_e4m3(y):
    """By search among the 127 magnitudes of the format (numpy)."""
    global _E4M3
    if _E4M3 is None:
        _E4M3 = np.array([m * 2.0 ** -9 for m in range(8)] + [(8 + m) * 2.0 ** (e - 10) for e in range(1, 16) for m in range(8)][:-1])
    a = np.abs(y)
    hi = np.clip(np.searchsorted(_E4M3, a), 1, len(_E4M3) - 1)
    lo = hi - 1
    below, above = a - _E4M3[lo], _E4M3[hi] - a
    i = np.where((below < above) | ((below == above) & (lo % 2 == 0)), lo, hi)
    return np.copysign(_E4M3[i], y)


def _value_rows(pool, scales, layer, page, head):
    """One head of pages as float64 [pages, rows, dim]."""
    x = pool[layer, page, head] if pool.dtype != torch.float8_e4m3fn else pool.view(torch.uint8)[layer, page, head].view(pool.dtype)
    x = x.to(torch.float32).double()
    return x if scales is None else x * scales[layer, page, head].double()[..., None]


def exact(case, seed):
    c, s = case, _inputs(case, seed)
    t = c.get("page_tokens", 1)
    if c["op"] == "append":
        table, seq, pos = (s[n].cpu().numpy() for n in ("tables", "seq", "pos"))
        page, row = torch.from_numpy(table[seq, pos // t]).long(), torch.from_numpy(pos % t).long()
        out = []
        for pool, scales, rows in ((s["k"], s["k_scale"], s["k_rows"]), (s["v"], s["v_scale"], s["v_rows"])):
            r = rows.double().cpu().numpy()
            values = pool.float().cpu().double()
            if c["store"] in TOP:
                sc = np.maximum((np.abs(r).max(-1) / TOP[c["store"]]).astype(np.float32), np.float32(LEAST_SCALE))
                y = r / sc.astype(np.float64)[..., None]
                y = np.rint(y) if c["store"] == "i8" else _nearest_e4m3(y)
                kept = scales.cpu().double()
                kept[0, page, :, row] = torch.from_numpy(sc.astype(np.float64))
                values[0, page, :, row] = torch.from_numpy(y)
                out += [values.to(torch.int8) if c["store"] == "i8" else values, kept]
            else:
                values[0, page, :, row] = torch.from_numpy(r)
                out.append(values)
        return out
    if c["op"] == "read":
        out = []
        for pool, scales in ((s["k"], s["k_scale"]), (s["v"], s["v_scale"])):
            x = torch.stack([_value_rows(pool, scales, 0, slice(None), h) for h in range(c["kv_heads"])], 2)   # [page, row, head, dim]
            page = s["tables"][s["seq"].long(), s["pos"].long().div(t, rounding_mode="floor")].long()
            out.append(x.reshape(-1, *x.shape[2:])[page * t + s["pos"].long() % t])
        return out
    if c["op"] == "attention":
        n, hk, g, d = c["n_seqs"], c["kv_heads"], c["group"], c["head_dim"]
        out = torch.zeros((n, hk * g, d), dtype=torch.float64, device=DEVICE)
        for i, length in enumerate(_lens(c)):
            if length == 0:
                continue
            page = s["tables"][i, :-(-length // t)].long()
            first = max(0, length - c["window"]) if c["window"] else 0
            for h in range(hk):
                k, v = (_value_rows(s[a], s[a + "_scale"], 0, page, h).reshape(-1, d)[first:length] for a in ("k", "v"))
                x = (s["q"][i, h * g:(h + 1) * g].double() @ k.T) * d ** -0.5
                out[i, h * g:(h + 1) * g] = torch.softmax(x, -1) @ v
        return out
    if c["op"] == "select":
        g, w, v = c["groups"], c["width"], c["vocab"]
        logits, start = s["logits"].double().cpu().numpy(), s["scores"].double().cpu().numpy()
        ended, eos = s["finished"].cpu().numpy(), s["eos"]
        tokens, parents, scores, done = (np.zeros((g, w), t_) for t_ in (np.int32, np.int32, np.float64, bool))
        for b in range(g):
            found = []
            for i in range(w):
                if ended[b, i]:
                    found.append((-start[b, i], i, eos))
                    continue
                x = logits[b, i]
                m = x.max()
                lse = m + np.log(np.exp(x - m).sum())
                first = np.argsort(-x, kind="stable")[:w]      # no more than w of one beam can be among the w best
                found += [(-(start[b, i] + x[j] - lse), i, int(j)) for j in first]
            for r, (score, i, j) in enumerate(sorted(found)[:w]):
                tokens[b, r], parents[b, r], scores[b, r], done[b, r] = j, i, -score, ended[b, i] or j == eos
        return [torch.from_numpy(x) for x in (tokens, parents, scores, done)]
    g, w, full, part = c["groups"], c["width"], c["ctx"] // t, c["ctx"] % t
    before, after, parents = (s[n].cpu().numpy() for n in ("before", "after", "parents"))
    pools = [x for x in (s["k"], s["k_scale"], s["v"], s["v_scale"]) if x is not None]
    wide = [x.float() for x in pools]
    old = [x.clone() for x in wide]
    for b in range(g):
        for i in range(w):
            p = b * w + int(parents[b, i])
            after[b * w + i, :full] = before[p, :full]
            for x, y in zip(wide, old):
                x[:, int(after[b * w + i, full]), :, :part] = y[:, int(before[p, full]), :, :part]
    wide = [x.to(torch.int8) if p.dtype == torch.int8 else x.double() for x, p in zip(wide, pools)]
    return [torch.from_numpy(after)] + wide
