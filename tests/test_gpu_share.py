"""Attention of rows that share the first positions of their contexts, against 64 bits row by row.  Whatever a row may not see is NaN."""
import math

import numpy as np
import pytest
import torch

import page_util as pu
from share_util import DEV, Shared, ints, queries

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def nnc():
    from paper_2512_21571_amd import binding
    binding.lib()
    return binding


@pytest.mark.parametrize("store", list(pu.STORES))
@pytest.mark.parametrize("rows", list(pu.ROWS))
@pytest.mark.parametrize("heads,group,dim,tokens", [(2, 4, 128, 16), (3, 1, 64, 7), (1, 16, 128, 1), (2, 5, 64, 24), (1, 20, 128, 64)])
def test_prefix_and_what_is_behind(nnc, store, rows, heads, group, dim, tokens):
    lens = [[40, 33, 41, 73, 0], [1, 17, 16, 100, 30], [5, 0, 1, 2, 64]]
    s = Shared(nnc, store, lens, [40, 17, 0], tokens, heads, dim)
    q = queries((3, 5, heads * group, dim), rows)
    out = s.run(q)
    assert (out[0, 4] == 0).all() and (out[2, 1] == 0).all()
    s.check(q, out, rows)
    assert torch.equal(out, s.run(q))                                     # the same call, the same bits
    s.check(q, s.run(q, max_len=100, max_own=83), rows)


@pytest.mark.parametrize("store", list(pu.STORES))
@pytest.mark.parametrize("rows", list(pu.ROWS))
@pytest.mark.parametrize("heads,group,dim,tokens,width", [(2, 4, 128, 16, 5), (1, 3, 64, 7, 1), (2, 8, 128, 24, 6), (1, 16, 64, 16, 3)])
def test_new_tokens_of_one_sequence(nnc, store, rows, heads, group, dim, tokens, width):
    """Row j of a sequence sees one position more than row j - 1; a row of length zero, rows in any order."""
    lens = [[n + j for j in range(width)] for n in (1, 31, 60)] + [list(range(width))[::-1]]
    s = Shared(nnc, store, lens, [0] * 4, tokens, heads, dim, drafts=True)
    q = queries((4, width, heads * group, dim), rows)
    s.check(q, s.run(q), rows)
    s.check(q, s.run(q, max_len=int(s.lens.max())), rows)


@pytest.mark.parametrize("store,rows", [("bf16", "bf16"), ("bf16", "f32"), ("f16", "f16"), ("f16", "f32"), ("i8", "bf16"), ("i8", "f32"), ("e4m3", "bf16"), ("e4m3", "f16"), ("f32", "f32")])
@pytest.mark.parametrize("dim", [128, 64])
@pytest.mark.parametrize("groups,width,heads,group,prefix", [(1, 70, 1, 5, 1000), (2, 33, 2, 1, 700), (1, 3, 8, 16, 2500), (3, 2, 1, 2, 1500)])
def test_many_rows_and_long_prefixes(nnc, store, rows, dim, groups, width, heads, group, prefix):
    """Several blocks of rows, several workgroups along the prefix, own positions of every length up to a few tiles."""
    rng = np.random.default_rng(3)
    lens = prefix + rng.integers(0, 200, (groups, width))
    lens[0, 0], lens[-1, -1] = prefix // 2, prefix
    s = Shared(nnc, store, lens, [prefix] * groups, 32, heads, dim, loud=2.0)
    q = queries((groups, width, heads * group, dim), rows, size=2.0)
    assert s.p.attention_shared_workspace(q, s.tables, s.lens_t, s.prefix_t) > 0
    s.check(q, s.run(q), rows)


@pytest.mark.parametrize("store,rows", [("bf16", "bf16"), ("i8", "f32"), ("f32", "f32"), ("f16", "f16")])
def test_long_drafts(nnc, store, rows):
    lens = [[4000 - 7 + j for j in range(8)], [300 + j for j in range(8)], [j for j in range(8)]]
    s = Shared(nnc, store, lens, [0] * 3, 16, 2, 128, drafts=True)
    q = queries((3, 8, 8, 128), rows)
    s.check(q, s.run(q), rows)


@pytest.mark.parametrize("store,rows", [("bf16", "bf16"), ("bf16", "f32"), ("f16", "f16"), ("e4m3", "bf16"), ("i8", "bf16"), ("f32", "f32")])
@pytest.mark.parametrize("drafts", [False, True])
@pytest.mark.parametrize("bad", [math.nan, math.inf])
def test_what_other_rows_see_does_not_reach_a_row(nnc, store, rows, drafts, bad):
    """A position whose K or V is no number: rows that end before it are as if it were not there, the others show it."""
    where = 45
    lens = [[44, 45, 46, 64, 47, 7]]
    s = Shared(nnc, store, lens, [64], 16, 2, 128, drafts=drafts)
    q = queries((1, 6, 8, 128), rows)
    clean = s.run(q)
    for which in ("k", "v"):
        back = s.p.read(1, s.tables, 0, where, n=1)
        y = [back[0].clone(), back[1].clone()]
        y[which == "v"][0, :, 3] = bad
        s.p.append(1, y[0], y[1], s.tables, 0, where)
        out = s.run(q)
        sees = (s.lens_t > where).tolist()[0]
        for w in range(6):
            if sees[w]:
                assert not torch.isfinite(out[0, w]).all(), (which, w)
            else:
                assert torch.equal(out[0, w], clean[0, w]), (which, w)
        s.p.append(1, back[0], back[1], s.tables, 0, where)
        assert torch.equal(s.run(q), clean) or store in ("i8", "e4m3")       # (8-bit rows may not come back to the bit)


@pytest.mark.parametrize("store", ["bf16", "i8", "f32"])
def test_wrong_lengths_and_missing_pages_are_nan(nnc, store):
    lens = [[100, 60, 31, 128], [100, 100, 100, 100], [100, 64, 65, 40]]
    s = Shared(nnc, store, lens, [64, 64, 64], 16, 2, 128)
    q = queries((3, 4, 4, 128), "f32")
    clean = s.run(q)
    assert not clean.isnan().any()
    nan = lambda out: out.isnan().flatten(2).all(-1).tolist()
    any_nan = lambda out: out.isnan().flatten(2).any(-1).tolist()
    # a page of the prefix, looked up through the first row: rows that end in front of it are untouched
    s.tables[0, 2] = s.p.n_pages
    out = s.run(q)
    assert nan(out)[0] == [True, True, False, True] and any_nan(out)[0] == [True, True, False, True] and not out[1:].isnan().any()
    s.tables[0, 2] = int(s.table[0, 2])
    # ... of a row's own, and one of the prefix in a row that is not the first: nobody looks at it
    s.tables[1, 2] = s.tables[7, 0] = -1
    s.tables[6, 5] = -5
    out = s.run(q)
    assert any_nan(out) == [[False] * 4, [False, False, True, False], [False] * 4] and nan(out)[1][2]
    assert torch.equal(out[0], clean[0])
    s.tables.copy_(ints(s.table))
    s.lens_t[0, 1], s.lens_t[2, 3], s.prefix_t[1] = -1, 129, -2
    out = s.run(q)
    assert nan(out) == any_nan(out) == [[False, True, False, False], [True] * 4, [False, False, False, True]]
    s.lens_t.copy_(ints(lens))
    s.prefix_t.copy_(ints([64, 64, 64]))
    out = s.run(q, max_len=100, max_own=36)                                # one row is longer than that
    assert nan(out) == any_nan(out) == [[False, False, False, True], [False] * 4, [False] * 4]
    out = s.run(q, max_own=0)                                              # nothing behind the prefix: who has something there is NaN
    assert nan(out) == any_nan(out) == [[True, False, False, True], [True] * 4, [True, False, True, False]]
    s.prefix_t[0] = 1 << 30                                                # (a prefix beyond every length: all of a row's positions are the group's)
    out = s.run(q[:, :, :, :], max_own=64)
    assert torch.isfinite(out[0, 2]).all()


@pytest.mark.parametrize("store,rows,heads,group,dim", [("bf16", "bf16", 2, 2, 128), ("f16", "f32", 1, 5, 64), ("e4m3", "bf16", 1, 3, 128), ("f32", "f32", 1, 12, 128), ("f32", "bf16", 3, 7, 64)])
def test_few_rows_with_long_contexts_of_their_own(nnc, store, rows, heads, group, dim):
    """Up to sixteen rows, and fp32: one walk over the shared positions and each sequence's, which a workgroup's share may begin or end in;
    sequences whose heads lie in two workgroups; far fewer positions than the call allows, so that most workgroups have none."""
    lens = [[700, 650, 1300], [3, 0, 640]]
    s = Shared(nnc, store, lens, [650, 600], 16, heads, dim)
    q = queries((2, 3, heads * group, dim), rows)
    out = s.run(q)
    s.check(q, out, rows)
    assert torch.equal(out, s.run(q))
    wide = torch.full((6, 4096), -1, dtype=torch.int32, device=DEV)
    wide[:, :s.tables.shape[1]] = s.tables
    assert s.p.attention_shared_workspace(q, wide, s.lens_t, s.prefix_t) > 0
    s.check(q, s.p.attention_shared(1, q, wide, s.lens_t, s.prefix_t), rows)
    assert s.p.attention_shared_workspace(q, s.tables, s.lens_t, s.prefix_t, max_len=1300, max_own=0) > 0
    short = torch.minimum(s.lens_t, s.prefix_t[:, None]).contiguous()     # nobody behind the prefix
    got = s.p.attention_shared(1, q, s.tables, short, s.prefix_t, max_own=0)
    assert torch.isfinite(got).all() and not torch.equal(got[0, 2], out[0, 2])


def test_no_rows_and_one_row(nnc):
    s = Shared(nnc, "bf16", [[20]], [20], 16, 2, 64)
    q = queries((1, 1, 4, 64), "bf16")
    s.check(q, s.run(q, max_own=0), "bf16")
    assert s.p.attention_shared(1, q[:0], s.tables[:0], s.lens_t[:0], s.prefix_t[:0]).shape == (0, 1, 4, 64)
    assert s.p.attention_shared_workspace(q, s.tables, s.lens_t, s.prefix_t, max_len=20, max_own=0) == 0
    for tables, prefix in ((s.tables[:0], s.prefix_t), (s.tables, None)):                  # a group without rows
        assert s.p.attention_shared(1, q[:, :0], tables, s.lens_t[:, :0].contiguous(), prefix).shape == (1, 0, 4, 64)


@pytest.mark.parametrize("rows", list(pu.ROWS))
def test_strides_and_scales(nnc, rows):
    """Queries inside a fused projection at an odd alignment, the output over them; scales of either sign and zero."""
    s = Shared(nnc, "bf16", [[40, 50, 60], [33, 20, 35]], [32, 32], 16, 2, 64)
    wide = queries((6, 12 * 64 + 5), rows)
    q = wide[:, 5:].view(6, 12, 64)[:, ::3].unflatten(0, (2, 3))
    out = s.run(q)
    s.check(q, out, rows)
    for scale in (-0.2, 0.0, 3.0):
        # the same rows one by one, by the attention of one row per sequence
        got, alone = s.run(q, scale=scale), s.p.attention(1, q.flatten(0, 1), effective(s), s.lens_t.view(-1), scale=scale)
        # two results that are each off by no more than check_row allows (scores up to 60: 2 x 72 x 2^-24 x 60 x 2 = 1e-3 at |v| <= 5)
        tol = 2 * (5e-3 + 5 * pu.HALF_ULP[rows])
        assert bool(((got.flatten(0, 1).float() - alone.float()).abs() <= tol).all()), scale
    kept = wide.clone()
    assert s.run(q, out=q) is q and torch.equal(q, out)
    mask = torch.zeros(12, dtype=torch.bool)
    mask[::3] = True
    assert torch.equal(wide[:, 5:].view(6, 12, 64)[:, ~mask], kept[:, 5:].view(6, 12, 64)[:, ~mask]) and torch.equal(wide[:, :5], kept[:, :5])


def effective(s):
    """Tables through which each row finds its whole context by itself (prefixes of full pages)."""
    t = s.tables.clone()
    width = s.lens.shape[1]
    for r in range(len(t)):
        n = int(s.prefix[r // width]) // s.p.page_tokens
        t[r, :n] = t[r // width * width, :n]
    return t


def test_offsets_past_32_bits(nnc):
    """A pool whose last page starts beyond 2^32 bytes and 2^31 elements."""
    pages = 17000
    p = nnc.Pages.empty(1, pages, 128, 16, 64, torch.float16, DEV)
    tables = ints(pages - 1 - np.arange(4).reshape(2, 2))
    for i in range(2):
        p.append(0, *[torch.randn((256, 16, 64), device=DEV) for _ in range(2)], tables, i, 0)
    small = nnc.Pages(p.k[:, -4:].clone(), p.v[:, -4:].clone())
    q = queries((2, 3, 32, 64), "f16")
    lens = ints([[200, 256, 130], [1, 128, 250]])
    assert torch.equal(p.attention_shared(0, q, tables, lens), small.attention_shared(0, q, tables - (pages - 4), lens))


def test_in_a_graph_on_another_stream_and_with_shared_workspaces(nnc):
    """Captured and replayed between eager calls of other lengths through the same workspace; on a stream of the caller's."""
    s = Shared(nnc, "bf16", [[300, 333, 310, 350]], [300], 16, 4, 128)
    q = queries((1, 4, 16, 128), "bf16")
    size = s.p.attention_shared_workspace(q, s.tables, s.lens_t, s.prefix_t)
    ws = torch.empty(size, dtype=torch.uint8, device=DEV)
    out, lens, prefix = torch.empty_like(q), s.lens_t.clone(), s.prefix_t.clone()
    want = s.run(q)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        s.p.attention_shared(1, q, s.tables, lens, prefix, out=out, workspace=ws)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(out, want)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        s.p.attention_shared(1, q, s.tables, lens, prefix, out=out, workspace=ws)
    for step in range(4):
        q.copy_(queries((1, 4, 16, 128), "bf16", seed=step))
        lens.copy_(ints([[300 - step, 333, 310 - 5 * step, 300 + step]]))
        out.fill_(7.0)
        g.replay()
        got = out.clone()
        eager = s.p.attention_shared(1, q, s.tables, lens, prefix, workspace=ws)
        assert torch.equal(got, eager), step
        torch.cuda.synchronize()


@pytest.mark.parametrize("store,rows", [("bf16", "bf16"), ("i8", "bf16"), ("e4m3", "bf16"), ("f16", "f16"), ("bf16", "f32"), ("f32", "bf16")])
@pytest.mark.parametrize("dim", [128, 64])
def test_weights_where_sums_cancel(nnc, store, rows, dim):
    """Sums that cancel to 2^-13 of their terms, as for the attention of one row: every row of a group sees the same six rows, its scores
    exact products, and what is left must be right to 2^-20 of the terms.  Two binary16 pieces of a weight leave 2^-22 more out (half a step, 2^-11,
    of half a step), two pieces of bf16, with bf16 rows over 16- and 8-bit pools, 2^-18 (2^-9 of 2^-9)."""
    from test_gpu_pages_precision import cancelling
    rng = np.random.default_rng(11)
    n, width = 6, 40
    p = nnc.Pages.empty(1, 1, 8, 1, dim, pu.STORES[store], DEV)
    s, v, scale = cancelling(rng, store, dim, n)
    k = np.zeros((n, dim))
    k[:, 0] = s
    vv, kk = np.zeros((8, dim)), np.zeros((8, dim))
    vv[:n], kk[:n] = v, k
    p.v.copy_(torch.from_numpy(vv).float()[None, None, None].to(p.v.dtype))
    if p.k_scale is None:
        p.k.copy_(torch.from_numpy(kk).float()[None, None, None].to(p.k.dtype))
    else:                                                                # (the row's scale is its score, its first value -1)
        one = np.zeros((8, dim))
        one[:, 0] = -1
        p.k.copy_(torch.from_numpy(one).float()[None, None, None].to(p.k.dtype))
        p.k_scale.zero_()
        p.k_scale[0, 0, 0, :n] = torch.from_numpy(-s).float()
        p.v_scale.fill_(1.0)
        p.v_scale[0, 0, 0, :n] = torch.from_numpy(scale).float()
    q = torch.zeros((1, width, 1, dim), device=DEV, dtype=pu.ROWS[rows])
    q[..., 0] = 1.0
    out = p.attention_shared(0, q, ints([[0]]), ints([[n] * width]), scale=1.0)
    w = np.exp(s - s.max())
    x = v * scale[:, None]
    want, size = (w @ x) / w.sum(), (w @ np.abs(x)) / w.sum()
    bound = 2.0 ** -20 + (2.0 ** -22 if store == "f16" and rows == "f16" else 2.0 ** -18 if store != "f32" and rows == "bf16" else 0)
    tol = bound * size + pu.HALF_ULP[rows] * (np.abs(want) + bound * size) + (2.0 ** -25 if rows == "f16" else 0)
    err = np.abs(pu.f64(out)[0, :, 0] - want)
    assert (err <= tol).all(), float((err - tol).max())
