"""Bounds of pages, the pages that a query picks by them, and attention over what was picked, against 64 bits."""
import math

import numpy as np
import pytest
import torch

import page_util as pu
import share_util as su
from share_util import DEV, check_row, ints, make_pool, queries

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def nnc():
    from paper_2512_21571_amd import binding
    binding.lib()
    return binding


def filled(nnc, store, lens, tokens, heads, dim, seed=1, spare=2):
    rng = np.random.default_rng(seed)
    per = max(1, -(-max(lens) // tokens))
    p = make_pool(nnc, store, 2, len(lens) * per + spare, tokens, heads, dim)
    tables = ints(rng.permutation(p.n_pages)[:len(lens) * per].reshape(len(lens), per))
    gen = torch.Generator(device=DEV).manual_seed(seed)
    for i, n in enumerate(lens):
        if n:
            loud = torch.exp(torch.randn((n, heads, 1), generator=gen, device=DEV))
            p.append(1, *[torch.randn((n, heads, dim), generator=gen, device=DEV) * loud for _ in range(2)], tables, i, 0)
    return p, tables


def same_bits(a, b):
    v = {2: torch.int16, 4: torch.int32}[a.element_size()]
    return torch.equal(a.view(v), b.view(v))


def check_bounds(p, bounds, old, tables, lens, since, layer=1):
    """Bounds of the named pages by numpy, all others as they were."""
    k, _ = pu.pool_values(p, layer)
    scaled = p.k_scale is not None
    untouched = np.ones(p.n_pages, bool)
    t, tb = p.page_tokens, tables.cpu().numpy()
    for i, n in enumerate(lens):
        for b in range(since[i] // t, -(-n // t)):
            page = tb[i, b]
            untouched[page] = False
            x = k[page, :, :min(t, n - b * t)]
            for got, want, up in ((bounds[0], x.min(1), False), (bounds[1], x.max(1), True)):
                want = su.bf16_towards(want, up) if scaled else want
                assert np.array_equal(pu.f64(got[layer, page]), want), (i, b)
    for a, b in zip(bounds, old):
        assert same_bits(a[0], b[0]) and same_bits(a[1][torch.from_numpy(untouched).to(DEV)], b[1][torch.from_numpy(untouched).to(DEV)])


@pytest.mark.parametrize("store", list(pu.STORES))
@pytest.mark.parametrize("heads,dim,tokens", [(3, 128, 16), (1, 64, 1), (5, 64, 24), (2, 128, 7), (1, 128, 300), (8, 64, 64)])
def test_bounds(nnc, store, heads, dim, tokens):
    lens = [0, 1, tokens, tokens + 1, 3 * tokens, 5 * tokens - 1]
    p, tables = filled(nnc, store, lens, tokens, heads, dim)
    bounds = p.empty_bounds()
    for x in bounds:
        x.fill_(7.0)
    old = [x.clone() for x in bounds]
    ln = ints(lens)
    p.bound(1, bounds, tables, ln)
    check_bounds(p, bounds, old, tables, lens, [0] * 6)
    # only what is new: the last page or two
    for new in (1, 2, tokens, tokens + 1):
        for x in bounds:
            x.fill_(7.0)
        since = [max(0, n - new) for n in lens]
        p.bound(1, bounds, tables, ln, since=ints(since), max_new=new if new <= tables.shape[1] * tokens else 0)
        check_bounds(p, bounds, old, tables, lens, since)
    for x in bounds:
        x.fill_(7.0)
    p.bound(1, bounds, tables, ln, since=tokens)
    check_bounds(p, bounds, old, tables, lens, [tokens] * 6)


@pytest.mark.parametrize("store", list(pu.STORES))
def test_bounds_of_keys_that_are_no_numbers_and_pages_that_are_not_there(nnc, store):
    p, tables = filled(nnc, store, [40, 40, 40], 16, 2, 64)
    bad = torch.ones((1, 2, 64), device=DEV)
    bad[0, 1, 5] = math.nan
    p.append(1, bad, bad, tables, 0, 20)
    bad[0, 1, 5] = math.inf
    p.append(1, bad, bad, tables, 1, 20)
    bounds = p.empty_bounds()
    for x in bounds:
        x.fill_(7.0)
    kept = int(tables[2, 1])
    tables[2, 1] = p.n_pages
    p.bound(1, bounds, tables, ints([40, 40, 40]))
    a, b = int(tables[0, 1]), int(tables[1, 1])
    scaled = store in pu.TOP
    for x in bounds:
        nan = x[1, a].isnan()
        assert nan[1, 5] and not nan[0].any() and (nan[1].all() if scaled else nan.sum() == 1)
        assert (x[1, kept] == 7).all()
    assert bounds[1][1, b, 1].isnan().all() if scaled else bounds[1][1, b, 1, 5] == math.inf
    for lens, since in ((ints([-1, -5, 0]), 0), (ints([40, 40, 40]), ints([-1, 40, 41]))):
        before = [x.clone() for x in bounds]
        p.bound(1, bounds, tables, lens, since=since)
        assert all(same_bits(x, y) for x, y in zip(bounds, before))


def test_bounds_round_outwards(nnc):
    """Products of a byte and a scale that lie next to a bf16 number, on it, between two, and below the smallest normal one."""
    rng = np.random.default_rng(3)
    for store in pu.TOP:
        p = make_pool(nnc, store, 1, 200, 1, 1, 64)
        vals = rng.integers(-127, 128, (200, 64)) if store == "i8" else np.sign(rng.standard_normal((200, 64))) * pu.E4M3[rng.integers(0, 127, (200, 64))]
        scale = np.exp(rng.uniform(-60, 20, 200)).astype(np.float32)
        near = (rng.integers(128, 256, 100) * 2.0 ** -7 * 2.0 ** rng.integers(-80, 10, 100)).astype(np.float32)
        scale[:100] = np.where(rng.random(100) < 0.5, near, np.nextafter(near, np.where(rng.random(100) < 0.5, np.float32(0), np.float32(np.inf))))
        p.k[0, :, 0, 0] = torch.from_numpy(vals).float().to(p.k.dtype).to(DEV)
        p.k_scale[0, :, 0, 0] = torch.from_numpy(scale).to(DEV)
        bounds = p.empty_bounds()
        p.bound(0, bounds, torch.arange(200, dtype=torch.int32, device=DEV)[None], ints([200]))
        x = vals * scale.astype(np.float64)[:, None]
        assert np.array_equal(pu.f64(bounds[0])[0, :, 0], su.bf16_towards(x, False)) and np.array_equal(pu.f64(bounds[1])[0, :, 0], su.bf16_towards(x, True))


# ---- picks -----------------------------------------------------------------------------------------------------

def random_bounds(p, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    lo, hi = p.empty_bounds()
    mid = torch.randn(lo.shape, generator=gen, device=DEV)
    half = torch.rand(lo.shape, generator=gen, device=DEV) + 0.2
    lo.copy_(mid - half)
    hi.copy_(mid + half)
    return lo, hi


def check_pick(p, got, bounds, q, tables, lens, keep, first, last, layer=1):
    lo, hi, qq, tb = pu.f64(bounds[0][layer]), pu.f64(bounds[1][layer]), pu.f64(q), tables.cpu().numpy()
    grp = q.shape[1] // p.n_kv_heads
    for i, n in enumerate(lens):
        for h in range(p.n_kv_heads):
            want, seen = su.pick(qq[i, h * grp:(h + 1) * grp], lo[:, h], hi[:, h], tb[i], n, p.page_tokens, keep, first, last)
            assert got[0][i, h].tolist() == want.tolist(), (i, h, n)
            assert int(got[1][i, h]) == seen


def pool_for(nnc, store, pages, tokens, heads, dim):
    t = pu.STORES[store]
    return make_pool(nnc, store, 2, pages, tokens, heads, dim)


@pytest.mark.parametrize("store", list(pu.STORES))
@pytest.mark.parametrize("rows", list(pu.ROWS))
@pytest.mark.parametrize("heads,group,dim,tokens", [(2, 4, 128, 16), (3, 1, 64, 7), (1, 16, 128, 1), (2, 5, 64, 24), (1, 2, 128, 16), (2, 2, 64, 24), (1, 1, 128, 5), (3, 3, 128, 16)])
def test_pick(nnc, store, rows, heads, group, dim, tokens):
    lens = [0, 1, tokens, 3 * tokens, 7 * tokens - (tokens > 1), 40 * tokens, 41 * tokens - tokens // 2]
    p = pool_for(nnc, store, 300, tokens, heads, dim)
    tables = ints(np.random.default_rng(2).permutation(300)[:7 * 41].reshape(7, 41))
    bounds, q = random_bounds(p, 3), queries((7, heads * group, dim), rows)
    ln = ints(lens)
    for keep, first, last in ((1, 0, 1), (5, 1, 2), (7, 0, 1), (40, 3, 3), (64, 1, 1)):
        got = p.pick(1, bounds, q, tables, ln, keep, first=first, last=last)
        check_pick(p, got, bounds, q, tables, lens, keep, first, last)
        again = p.pick(1, bounds, q, tables, ln, keep, first=first, last=last, max_len=max(lens))
        assert torch.equal(got[0], again[0]) and torch.equal(got[1], again[1])


@pytest.mark.parametrize("blocks,keep", [(1023, 7), (1024, 512), (1025, 1024), (5000, 100), (20000, 300), (2100, 2099)])
def test_pick_of_many_pages(nnc, blocks, keep):
    p = pool_for(nnc, "bf16", 9, 16, 2, 64)
    tables = ints(np.random.default_rng(blocks).integers(0, 9, (2, blocks)))      # few different pages: ties everywhere
    bounds, q = random_bounds(p, 4), queries((2, 4, 64), "bf16")
    lens = [blocks * 16, (blocks - 1) * 16 - 5]
    check_pick(p, p.pick(1, bounds, q, tables, ints(lens), keep, first=1, last=2), bounds, q, tables, lens, keep, 1, 2)
    p = pool_for(nnc, "bf16", blocks, 1, 1, 64)
    tables = ints(np.random.default_rng(1).permutation(blocks)[None])
    bounds, q = random_bounds(p, 5), queries((1, 3, 64), "f32")
    check_pick(p, p.pick(1, bounds, q, tables, ints([blocks]), keep), bounds, q, tables, [blocks], keep, 1, 1)


def test_ties_go_to_the_page_that_comes_first(nnc):
    p = pool_for(nnc, "f32", 50, 4, 2, 128)
    tables = ints(np.arange(50)[None])
    lo, hi = p.empty_bounds()
    q = torch.randn((1, 2, 128), device=DEV)
    for value in (0.0, -0.0, 1.0):
        lo.fill_(value)
        hi.fill_(value)
        got = p.pick(1, (lo, hi), q, tables, ints([200]), 9, first=0, last=2)
        assert got[0][0, 0].tolist() == list(range(7)) + [48, 49] and got[1].tolist() == [[36, 36]]
    lo[:, ::2], hi[:, ::2] = -0.0, -0.0                                       # zeros of both signs are equal
    lo[:, 1::2], hi[:, 1::2] = 0.0, 0.0
    assert p.pick(1, (lo, hi), q, tables, ints([200]), 9, first=0, last=2)[0][0, 1].tolist() == list(range(7)) + [48, 49]


def test_scores_that_lie_close(nnc):
    """Pages whose scores differ by 2^-40 of their terms are told apart."""
    p = pool_for(nnc, "f32", 64, 1, 1, 64)
    lo, hi = p.empty_bounds()
    lo.zero_()
    hi.zero_()
    order = np.random.default_rng(1).permutation(64)
    hi[1, :, 0, 0] = lo[1, :, 0, 0] = 1024.0
    hi[1, :, 0, 1] = lo[1, :, 0, 1] = torch.from_numpy(order.astype(np.float32) * 2.0 ** -30).to(DEV)
    q = torch.zeros((1, 1, 64), device=DEV)
    q[..., :2] = 1.0
    got = p.pick(1, (lo, hi), q, ints(np.arange(64)[None]), ints([64]), 20, first=0, last=1)
    want = sorted(np.argsort(-order)[:20].tolist())
    if 63 not in want:
        want = sorted(np.argsort(-order)[:19].tolist() + [63])
    assert got[0][0, 0].tolist() == want


def test_pages_that_are_not_there_and_scores_that_are_no_numbers_come_first(nnc):
    p = pool_for(nnc, "bf16", 40, 16, 2, 64)
    tables = ints(np.arange(40)[None].repeat(4, 0))
    lo, hi = random_bounds(p, 1)
    q = queries((4, 4, 64), "bf16")
    tables[0, 17], tables[0, 30] = -3, 40
    lo[1, 11, 1, 5] = math.nan
    hi[1, 13, 0] = math.inf
    ln = ints([640, 640, -1, 641])
    t, n = p.pick(1, (lo, hi), q, tables, ln, 6)
    assert {-3, 40, 0, 39} <= set(t[0, 0].tolist()) and 13 in t[0, 0].tolist() and 11 in t[0, 1].tolist()
    assert 13 in t[1, 0].tolist() and 11 in t[1, 1].tolist()
    assert (t[2:] == -1).all() and n.tolist() == [[96, 96], [96, 96], [-1, -1], [-1, -1]]
    out = p.attention(1, q, t, n)
    assert out[0].isnan().all() and out[2:].isnan().all()
    q[1, :2] = math.nan                                                       # a query that is no number: the first pages, the last one
    assert p.pick(1, (lo, hi), q, tables, ints([640] * 4), 6)[0][1, 0].tolist() == [0, 1, 2, 3, 4, 39]
    t, n = p.pick(1, (lo, hi), q, tables, ints([640, 33, 0, 640]), 6, max_len=100)
    assert n.tolist() == [[-1, -1], [33, 33], [0, 0], [-1, -1]] and t[1, 0].tolist() == [0, 1, 2, -1, -1, -1]


# ---- attention over what was picked ----------------------------------------------------------------------------

@pytest.mark.parametrize("store", list(pu.STORES))
@pytest.mark.parametrize("rows", list(pu.ROWS))
@pytest.mark.parametrize("heads,group,dim,tokens", [(2, 4, 128, 16), (3, 1, 64, 7), (1, 20, 128, 64), (2, 16, 64, 1)])
def test_bound_pick_and_attend(nnc, store, rows, heads, group, dim, tokens):
    """As a step does it: bounds, picks, attention; with all pages kept, that of the whole context, to the bit."""
    lens = [0, 1, 3 * tokens, 12 * tokens - tokens // 2, 20 * tokens]
    p, tables = filled(nnc, store, lens, tokens, heads, dim)
    bounds, q, ln = p.empty_bounds(), queries((5, heads * group, dim), rows), ints(lens)
    p.bound(1, bounds, tables, ln)
    t, n = p.pick(1, bounds, q, tables, ln, 5)
    out = p.attention(1, q, t, n)
    k, v = pu.pool_values(p, 1)
    got, qq, tb, seen = pu.f64(out), pu.f64(q), t.cpu().numpy(), n.cpu().numpy()
    for i in range(5):
        for h in range(heads):
            pos = np.arange(seen[i, h])
            page, s = tb[i, h][pos // tokens], slice(h * group, (h + 1) * group)
            check_row(p, got[i, s], qq[i, s], k[page, h, pos % tokens], v[page, h, pos % tokens], rows, (i, h))
    t, n = p.pick(1, bounds, q, tables, ln, tables.shape[1])
    assert (n == ln[:, None]).all()
    assert torch.equal(p.attention(1, q, t, n), p.attention(1, q, tables, ln))


def test_picked_attention_that_is_split(nnc):
    p, tables = filled(nnc, "bf16", [4000, 2500], 16, 2, 128)
    bounds, q, ln = p.empty_bounds(), queries((2, 8, 128), "bf16"), ints([4000, 2500])
    p.bound(1, bounds, tables, ln)
    t, n = p.pick(1, bounds, q, tables, ln, 100)
    assert p.attention_workspace(q, t, n) > 0
    k, v = pu.pool_values(p, 1)
    got, qq, tb = pu.f64(p.attention(1, q, t, n)), pu.f64(q), t.cpu().numpy()
    ws = torch.empty(p.attention_workspace(q, t, n), dtype=torch.uint8, device=DEV)
    assert torch.equal(p.attention(1, q, t, n, workspace=ws), p.attention(1, q, t, n))
    for i in range(2):
        for h in range(2):
            pos = np.arange(int(n[i, h]))
            check_row(p, got[i, h * 4:h * 4 + 4], qq[i, h * 4:h * 4 + 4], k[tb[i, h][pos // 16], h, pos % 16], v[tb[i, h][pos // 16], h, pos % 16], "bf16", (i, h))


def test_offsets_past_32_bits(nnc):
    """A pool whose last pages and whose bounds of them start beyond 2^32 bytes."""
    pages = 2200000
    p = nnc.Pages.empty(1, pages, 1, 16, 64, torch.float16, DEV)
    tables = ints(pages - 1 - np.arange(60).reshape(2, 30))
    for i in range(2):
        p.append(0, *[torch.randn((30, 16, 64), device=DEV) for _ in range(2)], tables, i, 0)
    bounds, q, ln = p.empty_bounds(), queries((2, 32, 64), "f16"), ints([30, 27])
    p.bound(0, bounds, tables, ln)
    small = nnc.Pages(p.k[:, -60:].clone(), p.v[:, -60:].clone())
    few, near = small.empty_bounds(), tables - (pages - 60)
    small.bound(0, few, near, ln)
    assert (pages - 60) * 16 * 64 * 2 > 2 ** 32
    for b, want in zip(bounds, few):
        assert torch.equal(b[0, pages - 60 + 3:], want[0, 3:])           # (the pages behind a sequence's end are left as they were)
    t, n = p.pick(0, bounds, q, tables, ln, 9)
    t2, n2 = small.pick(0, few, q, near, ln, 9)
    assert torch.equal(t - (pages - 60), t2) and torch.equal(n, n2)
    assert torch.equal(p.attention(0, q, t, n), small.attention(0, q, t2, n2))


def test_a_run_of_steps_in_a_graph(nnc):
    """Append, bounds of the new row's page, picks and attention, captured once and replayed as the sequences grow."""
    lens = [100, 37]
    p, tables = filled(nnc, "i8", [160, 160], 16, 2, 64)
    bounds, ln = p.empty_bounds(), ints(lens)
    p.bound(1, bounds, tables, ln)
    s = dict(k=torch.zeros((2, 2, 64), device=DEV), q=queries((2, 4, 64), "bf16"), seq=ints([0, 1]))
    ref_bounds = p.empty_bounds()

    def step(b):
        p.append(1, s["k"], s["k"], tables, s["seq"], ln)
        ln.add_(1)
        p.bound(1, b, tables, ln, since=ln - 1, max_new=1)
        t, n = p.pick(1, b, s["q"], tables, ln, 4, max_len=160)
        return t, n, p.attention(1, s["q"], t, n)

    keep = ln.clone()
    step(bounds)
    ln.copy_(keep)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = step(bounds)
    for i in range(6):
        s["k"].copy_(torch.randn((2, 2, 64), generator=torch.Generator(device=DEV).manual_seed(i), device=DEV))
        g.replay()
        p.bound(1, ref_bounds, tables, ln)
        t, n = p.pick(1, ref_bounds, s["q"], tables, ln, 4)
        torch.cuda.synchronize()
        assert torch.equal(out[0], t) and torch.equal(out[1], n) and torch.equal(out[2], p.attention(1, s["q"], t, n))
