"""What the weights of shared and of picked attention carry, in every form of their kernels, where sums cancel."""
import numpy as np
import pytest
import torch

import page_util as pu
from share_util import DEV, ints
from test_gpu_pages_precision import cancelling

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def nnc():
    from paper_2512_21571_amd import binding
    binding.lib()
    return binding


N = 6


def cancelling_pool(nnc, store, dim):
    """One page of eight rows, of which N are used: pool, scores, values as they are read."""
    s, v, scale = cancelling(np.random.default_rng(11), store, dim, N)
    p = nnc.Pages.empty(1, 1, 8, 1, dim, pu.STORES[store], DEV)
    k, x = np.zeros((8, dim)), np.zeros((8, dim))
    k[:N, 0], x[:N] = s, v
    p.v.copy_(torch.from_numpy(x).float()[None, None, None].to(p.v.dtype))
    if p.k_scale is None:
        p.k.copy_(torch.from_numpy(k).float()[None, None, None].to(p.k.dtype))
    else:                                                                    # (the row's scale is its score, its first value -1)
        k[:, 0] = -1
        p.k.copy_(torch.from_numpy(k).float()[None, None, None].to(p.k.dtype))
        p.k_scale.zero_()
        p.k_scale[0, 0, 0, :N] = torch.from_numpy(-s).float()
        p.v_scale.fill_(1.0)
        p.v_scale[0, 0, 0, :N] = torch.from_numpy(scale).float()
    return p, s, v * scale[:, None]


def check(out, s, x, rows, left_out):
    """Every row of out sees all N: below 15 x 2^-24 of the terms from scores, exponentials and sums (2^-20 is the bound), and what the weights' pieces leave out."""
    w = np.exp(s - s.max())
    want, size = (w @ x) / w.sum(), (w @ np.abs(x)) / w.sum()
    err = (2.0 ** -20 + left_out) * size
    tol = err + pu.HALF_ULP[rows] * (np.abs(want) + err) + (2.0 ** -25 if rows == "f16" else 0)
    off = np.abs(pu.f64(out).reshape(-1, out.shape[-1]) - want)
    assert (off <= tol).all(), float((off / tol).max())


@pytest.mark.parametrize("store,rows", [("bf16", "bf16"), ("i8", "bf16"), ("e4m3", "bf16"), ("f16", "f16"), ("bf16", "f32"), ("i8", "f32"), ("f16", "bf16"), ("f32", "bf16")])
@pytest.mark.parametrize("dim", [128, 64])
@pytest.mark.parametrize("width,prefix", [(1, 3), (4, 3), (4, None), (16, 0), (16, 6), (20, None), (20, 3), (40, 4), (64, None), (100, None), (100, 3), (130, None)])
def test_sums_that_cancel(nnc, store, rows, dim, width, prefix):
    """Rows behind a prefix (up to sixteen in one launch, more in two) and rows without positions of their own, in workgroups of 16, 32, 64 and
    128.  Two pieces of a weight leave 2^-22 (binary16) or, where the pool's products are in bf16 and so are the rows, 2^-18 of it out."""
    p, s, x = cancelling_pool(nnc, store, dim)
    q = torch.zeros((1, width, 1, dim), device=DEV, dtype=pu.ROWS[rows])
    q[..., 0] = 1.0
    lens = ints([[N] * width])
    if prefix is None:
        out = p.attention_shared(0, q, ints([[0]]), lens, scale=1.0)
    else:
        out = p.attention_shared(0, q, ints([[0]] * width), lens, ints([prefix]), max_own=N - prefix, scale=1.0)
    two = 2.0 ** -22 if store == rows == "f16" else 2.0 ** -18 if store in ("bf16", "i8", "e4m3") and rows == "bf16" else 0.0
    check(out, s, x, rows, two)


@pytest.mark.parametrize("store,rows", [("bf16", "bf16"), ("i8", "bf16"), ("e4m3", "bf16"), ("f16", "f16"), ("bf16", "f32"), ("f16", "bf16"), ("f32", "bf16")])
@pytest.mark.parametrize("dim", [128, 64])
def test_picked_pages_have_the_weights_of_one_row(nnc, store, rows, dim):
    p, s, x = cancelling_pool(nnc, store, dim)
    q = torch.zeros((3, 2, dim), device=DEV, dtype=pu.ROWS[rows])
    q[..., 0] = 1.0
    out = p.attention(0, q, ints([[[0]]] * 3), ints([[N]] * 3), scale=1.0)
    check(out, s, x, rows, 2.0 ** -22 if store == rows == "f16" else 0.0)


@pytest.mark.parametrize("store", ["bf16", "i8", "e4m3"])
@pytest.mark.parametrize("dim", [128, 64])
@pytest.mark.parametrize("width,prefix", [(1, 3), (1, 0), (4, 3), (8, 5), (16, 0)])
def test_up_to_sixteen_rows_with_their_own_positions_have_the_weights_of_one_row(nnc, store, dim, width, prefix):
    """Forty groups of different scores: what a weight's pieces leave out differs from score to score."""
    groups, rng = 40, np.random.default_rng(3)
    p = nnc.Pages.empty(1, groups, 8, 1, dim, pu.STORES[store], DEV)
    made = [cancelling(rng, store, dim, N) for _ in range(groups)]
    k, v, ks, vs = np.zeros((groups, 8, dim)), np.zeros((groups, 8, dim)), np.zeros((groups, 8)), np.ones((groups, 8))
    for i, (s, x, scale) in enumerate(made):
        k[i, :N, 0], v[i, :N], ks[i, :N], vs[i, :N] = (s if store == "bf16" else -1), x, -s, scale
    p.k.copy_(torch.from_numpy(k).float()[None, :, None].to(p.k.dtype))
    p.v.copy_(torch.from_numpy(v).float()[None, :, None].to(p.v.dtype))
    if p.k_scale is not None:
        p.k_scale.copy_(torch.from_numpy(ks).float()[None, :, None])
        p.v_scale.copy_(torch.from_numpy(vs).float()[None, :, None])
    q = torch.zeros((groups, width, 1, dim), device=DEV, dtype=torch.bfloat16)
    q[..., 0] = 1.0
    out = p.attention_shared(0, q, ints(np.repeat(np.arange(groups), width)[:, None]), ints(np.full((groups, width), N)), ints(np.full(groups, prefix)), max_own=N - prefix, scale=1.0)
    for i, (s, x, scale) in enumerate(made):
        check(out[i], s, x * scale[:, None], "bf16", 0.0)
