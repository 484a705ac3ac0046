"""What the paged attention's weights carry, seen where the output is next to nothing and their error is not."""
import numpy as np
import pytest
import torch

import page_util as pu

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def nnc():
    from paper_2512_21571_amd import binding
    binding.lib()
    return binding


def near(x, store):
    """float64 -> the nearest value of a stored format (8-bit formats: scale 1)."""
    if store == "e4m3":
        return pu.nearest_e4m3(np.clip(x, -448, 448))
    return pu.f64(torch.from_numpy(x).to(pu.STORES[store]))


def cancelling(rng, store, dim, n):
    """Scores (numbers of bf16 and binary16) and rows of V whose weighted sum is next to nothing in every dim: the first row is
    random, each of the others takes away what the rows before it have left.  int8 rows have scales that fall as what is left does."""
    s = -np.array([0.0] + [rng.integers(1, 90) / 128.0] + [2.0 * j for j in range(1, n - 1)])
    w = np.exp(s)
    scale = np.array([2.0 ** (-6 - 4 * max(0, j - 1)) for j in range(n)]) if store == "i8" else np.ones(n)
    v, left = np.zeros((n, dim)), np.zeros(dim)
    for j in range(n):
        want = (rng.uniform(0.4, 0.6, dim) * rng.choice([-1, 1], dim) if j == 0 else -left / w[j]) / scale[j]
        v[j] = np.clip(np.rint(want), -127, 127) if store == "i8" else near(want, store)
        left = left + w[j] * v[j] * scale[j]
    return s, v, scale


@pytest.mark.parametrize("dim", [128, 64])
@pytest.mark.parametrize("store,rows", [("bf16", "bf16"), ("i8", "bf16"), ("e4m3", "bf16"), ("f16", "f16"), ("bf16", "f32"), ("e4m3", "f16"), ("f32", "bf16")])
def test_weights_are_as_good_as_fp32(nnc, store, rows, dim):
    """Sums that cancel to 2^-13 of their terms and less, so that the output's own rounding is below the terms' 2^-21.  A score here is one product
    (exact); its multiple in base 2 is off by 2^-23 of at most 1.02 for the two large weights (two roundings), the difference from the maximum by 2^-24, the exponential by
    2^-23, a weight times a row's scale by 2^-24, sums of 6 terms by 6 x 2^-24, the
    quotient by 2^-24: below 15 x 2^-24 of sum w |v| / sum w in all, and the bound is 2^-20.  (The later weights' larger scores belong to
    terms that are smaller by as much.)  Two binary16 pieces of a weight leave 2^-22 of it out, which is added for that pool."""
    rng = np.random.default_rng(11)
    n_seqs, n = 48, 6
    p = nnc.Pages.empty(1, n_seqs, 8, 1, dim, pu.STORES[store], DEV)
    k, v, scales = np.zeros((n_seqs, 8, dim)), np.zeros((n_seqs, 8, dim)), np.ones((n_seqs, 8))
    for i in range(n_seqs):
        s, x, sc = cancelling(rng, store, dim, n)
        k[i, :n, 0] = s
        v[i, :n], scales[i, :n] = x, sc
    kept = torch.from_numpy(v).float()
    p.v.copy_(kept[None, :, None].to(p.v.dtype))
    if p.k_scale is None:
        p.k.copy_(torch.from_numpy(k).float()[None, :, None].to(p.k.dtype))
    else:                                                                # (the row's scale is its score, its first value -1)
        p.k.copy_(torch.from_numpy(np.sign(k)).float()[None, :, None].to(p.k.dtype))
        p.k_scale.copy_(torch.from_numpy(np.where(k[:, :, 0] == 0, 1.0, -k[:, :, 0])).float()[None, :, None])
        p.v_scale.copy_(torch.from_numpy(scales).float()[None, :, None])
    tables = torch.arange(n_seqs, dtype=torch.int32, device=DEV)[:, None]
    q = torch.zeros((n_seqs, 2, dim), device=DEV, dtype=pu.ROWS[rows])
    q[:, :, 0] = 1
    out = pu.f64(p.attention(0, q, tables, torch.full((n_seqs,), n, dtype=torch.int32, device=DEV), scale=1.0))
    kv, vv = pu.pool_values(p)
    worst = 0.0
    for i in range(n_seqs):
        w = np.exp(kv[i, 0, :n, 0])
        want, size = w @ vv[i, 0, :n] / w.sum(), w @ np.abs(vv[i, 0, :n]) / w.sum()
        assert (np.abs(want) <= 2.0 ** -13 * size).mean() > 0.9           # the sums do cancel
        err = (2.0 ** -20 + (2.0 ** -22 if store == "f16" else 0)) * size
        tol = err + pu.HALF_ULP[rows] * (np.abs(want) + err) + (2.0 ** -25 if rows == "f16" else 0)
        worst = max(worst, float((np.abs(out[i] - want) / tol).max()))
    assert worst <= 1.0, worst
