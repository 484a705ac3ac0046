"""Plain 64-bit definitions of the operators beside a paged cache for the tests: rows that share positions, verification of
drafts, bounds and picks (numpy; nothing of the library in here)."""
import math

import numpy as np
import torch

import page_util as pu

DEV = "cuda:0"


def make_pool(nnc, store, layers=1, pages=12, tokens=16, heads=3, dim=128):
    """Every value a NaN (int8: -128, which is never stored; its scale is a NaN)."""
    p = nnc.Pages.empty(layers, pages, tokens, heads, dim, pu.STORES[store], DEV)
    for x in (p.k, p.v):
        x.view(torch.uint8).fill_(0x80 if store == "i8" else 0xff)
    for x in (p.k_scale, p.v_scale):
        if x is not None:
            x.fill_(math.nan)
    return p


def ints(x):
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.int32)).to(DEV)


def row_bound(p, rows, size, n, top):
    """How far a row of attention over n positions may be off, per unit of the largest |v| (top): an fp32 score of head_dim products by (dim + 8)
    2^-24 of the sum of their magnitudes, size (twice: weight and normaliser), exponentials 2^-22, weights in pieces 2^-22, sums of n terms n 2^-24.
    With bf16 rows a weight is two pieces of bf16: the first leaves 2^-9 of it at most, the second 2^-9 of that, so that a sum of weighted values
    is off by 2^-18 of the largest (of this bound, which is taken twice, half)."""
    return 2 * (p.head_dim + 8) * 2.0 ** -24 * size + 2.0 ** -21 + (n + 64) * 2.0 ** -24 + (2.0 ** -19 if rows == "bf16" else 0)


def check_row(p, got, q, k, v, rows, what):
    """One row [heads of a kv head, dim] of an attention against 64 bits, then one rounding of the output."""
    want, size = pu.attention(q, k, v, p.head_dim ** -0.5)
    top = np.abs(v).max() if len(v) else 0.0
    rel = 2 * top * row_bound(p, rows, size, len(v), top)
    tol = rel + pu.HALF_ULP[rows] * (np.abs(want) + rel) + (2.0 ** -25 if rows == "f16" else 0)
    err = np.abs(got - want)
    assert (err <= tol).all(), (what, float((err - tol).max()), float(err.max()))


class Shared:
    """Groups of rows over a pool in which everything that no row may see is NaN.  lens [groups][width], prefix [groups]; drafts: a row of
    the table for each group, all of whose positions are there."""

    def __init__(self, nnc, store, lens, prefix, tokens, heads, dim, drafts=False, seed=1, loud=1.0):
        rng = np.random.default_rng(seed)
        self.lens, self.prefix, self.drafts = np.array(lens), np.array(prefix), drafts
        groups, width = self.lens.shape
        blocks = lambda n: -(-int(n) // tokens)
        most = max(1, max(blocks(n) for n in self.lens.flat))
        need = groups * most * (2 if drafts else width + 1) + 1
        self.p = p = make_pool(nnc, store, 2, need, tokens, heads, dim)
        free = rng.permutation(need).tolist()
        table = np.full((groups if drafts else groups * width, most), -1, np.int32)
        gen = torch.Generator(device=DEV).manual_seed(seed)

        def rows(n):
            return [torch.randn((n, heads, dim), generator=gen, device=DEV) * loud for _ in range(2)]

        for g in range(groups):
            top = int(self.lens[g].max())
            mine = [g] if drafts else range(g * width, (g + 1) * width)
            shared = top if drafts else int(min(prefix[g], top))
            first = [free.pop() for _ in range(blocks(shared))]
            for i, r in enumerate(mine):
                n = top if drafts else int(self.lens[g, r - g * width])
                full = shared // tokens
                table[r, :blocks(n)] = (first[:full] + [free.pop() for _ in range(most)])[:blocks(n)]
                if i == 0:
                    table[r, :len(first)] = first
                    if shared:
                        p.append(1, *rows(shared), ints(table), r, 0)
                if not drafts and n > prefix[g]:     # its own positions (what it has in front of them is never read, but through row 0)
                    p.append(1, *rows(n - int(prefix[g])), ints(table), r, int(prefix[g]))
        self.table = table
        self.tables, self.lens_t, self.prefix_t = ints(table), ints(self.lens), ints(self.prefix)

    def context(self, g, w, values, h):
        """k, v of a row's positions as the definition reads them."""
        t, width = self.p.page_tokens, self.lens.shape[1]
        pos = np.arange(max(0, int(self.lens[g, w])))
        if self.drafts:
            page = self.table[g][pos // t]
        else:
            page = np.where(pos < self.prefix[g], self.table[g * width][pos // t], self.table[g * width + w][pos // t])
        return [x[page, h, pos % t] for x in values]

    def check(self, q, out, rows):
        values = pu.pool_values(self.p, 1)
        got, qq = pu.f64(out), pu.f64(q)
        grp = q.shape[2] // self.p.n_kv_heads
        for g in range(q.shape[0]):
            for w in range(q.shape[1]):
                for h in range(self.p.n_kv_heads):
                    s = slice(h * grp, (h + 1) * grp)
                    check_row(self.p, got[g, w, s], qq[g, w, s], *self.context(g, w, values, h), rows, (g, w, h, int(self.lens[g, w])))

    def run(self, q, **kw):
        if self.drafts:
            return self.p.attention_shared(1, q, self.tables, self.lens_t, **kw)
        return self.p.attention_shared(1, q, self.tables, self.lens_t, self.prefix_t, **kw)


def queries(shape, rows, seed=5, size=1.5):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    return (torch.randn(shape, generator=gen, device=DEV) * size).to(pu.ROWS[rows])


# ---- verification --------------------------------------------------------------------------------------------------

def softmax(x, t):
    if t == 0:
        return (np.arange(len(x)) == int(np.argmax(x))).astype(np.float64)
    e = np.exp((x - x.max()) / t)
    return e / e.sum()


def no_distribution(x):
    return bool(np.isnan(x).any() or not np.isfinite(x.max()))


def verify(logits, drafts, uniforms, draft_logits, counts, heat):
    """float64 arrays -> tokens, accepted, and the smallest distance of a decision from its border (relative to 1)."""
    n, rows, v = logits.shape
    tokens, accepted, near = np.full((n, rows), -1, np.int32), np.zeros(n, np.int32), 1.0
    for i in range(n):
        count, t, j = (rows - 1 if counts is None else int(counts[i])), float(heat[i]), 0
        if not 0 <= count < rows or not 0 <= t < math.inf:
            continue
        while True:
            bad = no_distribution(logits[i, j])
            if j < count:
                x = int(drafts[i, j])
                bad = bad or not 0 <= x < v or np.isnan(uniforms[i, j]) or (draft_logits is not None and no_distribution(draft_logits[i, j]))
            if bad or (j == count and np.isnan(uniforms[i, -1])):
                break
            r = p = softmax(logits[i, j], t)
            if j < count:
                q = (np.arange(v) == x).astype(np.float64) if draft_logits is None else softmax(draft_logits[i, j], t)
                if p[x] != 0:
                    near = min(near, abs(uniforms[i, j] * q[x] - p[x]) / p[x])
                if uniforms[i, j] * q[x] < p[x]:
                    tokens[i, j], j = x, j + 1
                    continue
                if np.isnan(uniforms[i, -1]):
                    bad = True
                    break
                r = np.maximum(p - q, 0)
                r = r if r.sum() > 0 else p
            sums = np.cumsum(r)
            goal = uniforms[i, -1] * sums[-1]
            near = min(near, np.abs(sums[:-1][r[1:] > 0] - goal).min(initial=sums[-1]) / sums[-1])
            tokens[i, j] = int(np.searchsorted(sums, goal, side="right"))
            break
        accepted[i] = j
    return tokens, accepted, near


# ---- bounds and picks ------------------------------------------------------------------------------------------------

def bf16_towards(x, up):
    """float64 -> the nearest bf16 that is not below (above) x: a step of bf16 is 2^-7 of the power of two below (subnormals: 2^-133)."""
    with np.errstate(invalid="ignore"):
        e = np.maximum(np.frexp(x)[1], -125)
        step = np.ldexp(1.0, e - 8)
        return (np.ceil if up else np.floor)(x / step) * step


def pick(q, lo, hi, table, length, tokens, keep, first, last):
    """q [query heads of a kv head, dim], lo, hi [page, dim] (float64) of one kv head -> pages (keep of them, -1 behind), positions."""
    out = np.full(keep, -1, np.int32)
    blocks = -(-length // tokens)
    if length == 0:
        return out, 0
    score = np.empty(blocks)
    for b in range(blocks):
        page = table[b]
        score[b] = np.nan
        if 0 <= page < len(lo):
            with np.errstate(invalid="ignore"):
                score[b] = max((np.maximum(x * lo[page], x * hi[page]).sum() for x in q), key=lambda s: math.inf if s != s else s)
    always = [b for b in range(blocks) if b < first or b >= blocks - last]
    order = always + sorted((b for b in range(blocks) if b not in set(always)), key=lambda b: (not np.isnan(score[b]), -score[b] if score[b] == score[b] else 0, b))
    chosen = sorted(order[:keep])
    out[:len(chosen)] = table[chosen]
    return out, (len(chosen) - 1) * tokens + length - (blocks - 1) * tokens
