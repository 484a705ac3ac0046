"""Bounds of pages without new positions."""
import pytest

import page_util as pu
from share_util import ints
from test_gpu_pick import check_bounds, filled, nnc  # noqa: F401

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
