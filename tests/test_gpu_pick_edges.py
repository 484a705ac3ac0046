"""Bounds of pages without new positions and with scales that are infinite, picks by infinite bounds and of thousands of pages."""
import math

import numpy as np
import pytest
import torch

import page_util as pu
from share_util import DEV, ints, make_pool, queries
from test_gpu_pick import check_bounds, check_pick, filled, nnc, random_bounds  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("store", list(pu.STORES))
def test_sequences_without_new_positions_leave_bounds_alone(nnc, store):
    """since at the length, or behind it: nothing of that sequence is brought up to date, the page of its last position no more than others, which another
    sequence, that sees more of it, may name as well."""
    lens = [40, 37, 33, 48]
    p, tables = filled(nnc, store, [48, 48, 48, 48], 16, 2, 64)
    bounds = p.empty_bounds()
    for x in bounds:
        x.fill_(7.0)
    old = [x.clone() for x in bounds]
    p.bound(1, bounds, tables, ints(lens), since=ints([40, 38, 47, 47]))
    check_bounds(p, bounds, old, tables, lens, [48, 48, 48, 47])             # (the last one's last page)
    for x in bounds:
        x.fill_(7.0)
    p.bound(1, bounds, tables, ints(lens), since=40, max_new=8)              # a number for all: only the longest has more
    check_bounds(p, bounds, old, tables, lens, [48, 48, 48, 40])
    shared = tables[3:].repeat(4, 1).contiguous()                            # all name the same pages, one has new positions
    for x in bounds:
        x.fill_(7.0)
    p.bound(1, bounds, shared, ints(lens), since=ints([40, 37, 33, 47]), max_new=1)
    check_bounds(p, bounds, old, shared, lens, [48, 48, 48, 47])


@pytest.mark.parametrize("store", list(pu.TOP))
@pytest.mark.parametrize("tokens", [1, 7, 40])
def test_bounds_of_rows_with_infinite_scales(nnc, store, tokens):
    """An infinite scale makes its row's zeros NaN and its other values infinite."""
    p, tables = filled(nnc, store, [3 * tokens], tokens, 2, 128)
    rng = np.random.default_rng(2)
    page = int(tables[0, 1])
    row = rng.integers(-1, 2, 128)                                            # (a third of them zeros)
    p.k[1, page, 1, tokens // 2] = torch.from_numpy(row).float().to(p.k.dtype).to(DEV)
    p.k_scale[1, page, 1, tokens // 2] = math.inf
    bounds = p.empty_bounds()
    p.bound(1, bounds, tables, ints([3 * tokens]))
    with np.errstate(invalid="ignore"):
        k = pu.pool_values(p, 1)[0][page, 1]
    lo, hi = (pu.f64(x[1, page, 1]) for x in bounds)
    assert np.array_equal(np.isnan(lo), row == 0) and np.array_equal(np.isnan(hi), row == 0)
    assert (hi[row > 0] == math.inf).all() and (lo[row < 0] == -math.inf).all()
    assert (lo[row > 0] <= k[:, row > 0].min(0)).all() and (hi[row < 0] >= k[:, row < 0].max(0)).all()


@pytest.mark.parametrize("store", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows", ["f32", "bf16"])
@pytest.mark.parametrize("heads,group,dim", [(1, 1, 128), (2, 2, 64), (2, 5, 128), (1, 4, 64)])
def test_scores_of_infinite_bounds(nnc, store, rows, heads, group, dim):
    """max(q lo, q hi) of an infinite bound is the other one's product where q has the sign for it, infinite where it has not, NaN where q is zero."""
    p = make_pool(nnc, store, 2, 60, 16, heads, dim)
    tables = ints(np.random.default_rng(1).permutation(60)[None].repeat(3, 0))
    bounds, q = random_bounds(p, 3), queries((3, heads * group, dim), rows)
    lo, hi = bounds
    q[0, :, 5], q[1, :, 5], q[2, :, 5] = 1.5, -1.5, 0.0
    q[:, :, 9] = -q[:, :, 5]
    lo[1, 10:20, :, 5] = -math.inf
    hi[1, 20:30, :, 5] = math.inf
    lo[1, 25:35, :, 9], hi[1, 25:35, :, 9] = -math.inf, math.inf
    lo[1, 40, :, 5], hi[1, 41, :, 9] = math.inf, -math.inf
    hi[1, 40, :, 5], lo[1, 41, :, 9] = math.inf, -math.inf
    lens = [960, 955, 960]
    for keep in (3, 12, 30, 50):
        check_pick(p, p.pick(1, bounds, q, tables, ints(lens), keep), bounds, q, tables, lens, keep, 1, 1)
    many = ints(np.random.default_rng(2).integers(0, 60, (3, 400)))          # the same pages beside infinite ones and beside others: ties everywhere
    lens = [6400, 6391, 6400]
    check_pick(p, p.pick(1, bounds, q, many, ints(lens), 150), bounds, q, many, lens, 150, 1, 1)
    lens = [960, 955, 960]
    lo[1, :, :, 5] = -math.inf                                               # on every page: only where q is positive does the score stay a number
    check_pick(p, p.pick(1, bounds, q, tables, ints(lens), 20), bounds, q, tables, lens, 20, 1, 1)


@pytest.mark.parametrize("store", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("heads,group,dim", [(1, 1, 128), (2, 2, 64), (2, 5, 128)])
def test_a_nan_in_one_bound_is_a_score_of_nan(nnc, store, heads, group, dim):
    """... whatever sign the query has there."""
    p = make_pool(nnc, store, 2, 60, 16, heads, dim)
    tables = ints(np.random.default_rng(1).permutation(60)[None].repeat(2, 0))
    bounds, q = random_bounds(p, 3), queries((2, heads * group, dim), "f32")
    q[0, :, 7], q[1, :, 7] = 0.5, -0.5
    bounds[0][1, 20, :, 7], bounds[1][1, 30, :, 7] = math.nan, math.nan
    bounds[0][1, 40, :, 3], bounds[1][1, 40, :, 4] = -math.inf, math.nan
    for keep in (3, 5, 20):
        check_pick(p, p.pick(1, bounds, q, tables, ints([960, 960]), keep), bounds, q, tables, [960, 960], keep, 1, 1)


@pytest.mark.parametrize("blocks,keep,first,last", [(8192, 256, 1, 2), (8193, 500, 2, 1), (12001, 64, 0, 1), (16384, 4096, 3, 9), (16385, 100, 1, 1)])
def test_pick_of_thousands_of_pages(nnc, blocks, keep, first, last):
    """Both sides of the number of pages that a thread keeps in registers, with ties and without."""
    p = make_pool(nnc, "bf16", 2, 50, 4, 1, 64)
    tables = ints(np.random.default_rng(blocks).integers(0, 50, (2, blocks)))
    bounds, q = random_bounds(p, 4), queries((2, 2, 64), "bf16")
    lens = [blocks * 4, blocks * 4 - 1021]
    check_pick(p, p.pick(1, bounds, q, tables, ints(lens), keep, first=first, last=last), bounds, q, tables, lens, keep, first, last)
    p = make_pool(nnc, "f16", 2, blocks, 1, 1, 64)
    tables = ints(np.random.default_rng(1).permutation(blocks)[None])
    bounds, q = random_bounds(p, 5), queries((1, 3, 64), "f32")
    check_pick(p, p.pick(1, bounds, q, tables, ints([blocks]), keep, first=first, last=last), bounds, q, tables, [blocks], keep, first, last)
