"""Verification of drafts at temperatures near zero and near the largest number, where a row's chunks have several pieces, where logits run
away along a row and where they lie at the end of their type, against the definition in 64 bits."""
import math

import numpy as np
import pytest
import torch

import page_util as pu
import share_util as su
from share_util import DEV, ints

pytestmark = pytest.mark.gpu

LOWEST = float(torch.finfo(torch.float32).min)


@pytest.fixture(scope="module")
def nnc():
    from paper_2512_21571_amd import binding
    binding.lib()
    return binding


def drawn(x, t, u):
    """One token of softmax(x / t) for a random number."""
    sums = np.cumsum(su.softmax(x, t))
    return int(np.searchsorted(sums, u * sums[-1], side="right"))


def inputs(n, k, v, rows, t, seed, size=2.5):
    """Drafts drawn at the temperature itself; targets that equal the draft's logits, differ from them by about the temperature (so that
    a draft may be kept or not), or by more."""
    rng = np.random.default_rng(seed)
    draft = torch.from_numpy(rng.standard_normal((n, k, v), dtype=np.float32) * np.float32(size)).to(pu.ROWS[rows])
    target = torch.from_numpy(rng.standard_normal((n, k + 1, v), dtype=np.float32) * np.float32(size)).to(pu.ROWS[rows])
    for i in range(n):
        noise = torch.from_numpy(rng.standard_normal((k, v), dtype=np.float32))
        target[i, :k] = (draft[i].float() + noise * (0.0, t, 0.5)[i % 3]).to(pu.ROWS[rows])
    u = rng.random((n, k + 1)).astype(np.float32).clip(0, 1 - 2.0 ** -24)
    drafts = np.array([[drawn(pu.f64(draft[i, j]), float(np.float32(t)), rng.random()) for j in range(k)] for i in range(n)], np.int32).reshape(n, k)
    return target, drafts, u, draft


def margin(logits, drafts, u, draft_logits, t):
    """How far the decisions of a call are from their borders.  p and q are good to 2^-41 of themselves (exponentials 2^-42 each way), so u q < p is
    certain beyond 2^-40 of the larger side, and a running sum of max(p - q, 0), whose terms are off by 2^-41 (p + q), beyond 2^-39."""
    n, rows, _ = logits.shape
    near = 1.0
    for i in range(n):
        for j in range(rows):
            r = p = su.softmax(logits[i, j], t)
            if j < rows - 1:
                x = int(drafts[i, j])
                q = su.softmax(draft_logits[i, j], t) if draft_logits is not None else (np.arange(len(p)) == x).astype(np.float64)
                a, b = float(u[i, j]) * q[x], p[x]
                if max(a, b) > 0:
                    near = min(near, abs(a - b) / max(a, b))
                if a < b:
                    continue
                r = np.maximum(p - q, 0)
                r = r if r.sum() > 0 else p
            sums = np.cumsum(r)
            near = min(near, np.abs(sums[:-1][r[1:] > 0] - float(u[i, -1]) * sums[-1]).min(initial=1.0))
            break
    return near


def check(nnc, target, drafts, u, draft, t):
    t = float(np.float32(t))
    dev = [torch.from_numpy(x).to(DEV) for x in (drafts, u)]
    heat = [np.float32(t)] * len(u)
    x, y = pu.f64(target), None if draft is None else pu.f64(draft)
    assert margin(x, drafts, u, y, t) > 2.0 ** -39
    want = su.verify(x, drafts, u.astype(np.float64), y, None, heat)
    got = nnc.draft_verify(target.to(DEV), *dev, None if draft is None else draft.to(DEV), temperature=t)
    assert np.array_equal(got[1].cpu().numpy(), want[1]) and np.array_equal(got[0].cpu().numpy(), want[0]), (t, draft is None)
    return want


# (pieces of 1024 a chunk: 1, 2, 3 and 4)
LOW = [shape + (t,) for t in (0.001, 0.005, 0.01, 0.05)
       for shape in ((2, 4, 151936, "f32"), (1, 4, 300001, "bf16"), (16, 5, 151936, "f32"), (64, 7, 35001, "f16"), (40, 3, 100003, "f32"))]


@pytest.mark.parametrize("n,k,v,rows,t", LOW + [(64, 7, 151936, "bf16", 0.005)])
def test_low_temperatures(nnc, n, k, v, rows, t):
    target, drafts, u, draft = inputs(n, k, v, rows, t, seed=v + k)
    check(nnc, target, drafts, u, draft, t)
    best = pu.f64(target[:, :k]).argmax(-1).astype(np.int32)
    check(nnc, target, best, u, None, t)


@pytest.mark.parametrize("v", [5003, 300001])
@pytest.mark.parametrize("t,step", [(1.0, 277.0), (1.0, 200.0), (1.0, 400.0), (1e-3, 0.3), (1e30, 2e32)])
def test_logits_that_run_away(nnc, v, t, step):
    """Logits that rise along the row by hundreds of temperatures, so that what was added up first is nothing beside what follows: 0, step,
    2 step in places that are one chunk's or several's; p is on the last one, two equal ones share it."""
    none = np.zeros((4, 0), np.int32)
    u = np.array([[0.001], [0.4], [0.6], [0.999]], np.float32)
    for places in ((3, 1030, 2900), (100, 1023, 1024), (10, 20, 2047), (v // 2, v // 2 + 1200, v - 1), (5, v - 2, v - 1)):
        for last in (2.0, 1.0):
            x = np.zeros((4, 1, v), np.float32)
            x[..., places[1]] = step
            x[..., places[2]] = step * last
            want = check(nnc, torch.from_numpy(x), none, u, None, t)
            assert (want[0][:, 0] == (places[2] if last == 2 else np.array([places[1]] * 2 + [places[2]] * 2))).all()


@pytest.mark.parametrize("t", [1.2e36, 1.3e36, 1e37, 3.4028234e38])
@pytest.mark.parametrize("n,k,v", [(3, 2, 777), (2, 3, 5003), (1, 2, 300001), (40, 3, 100003)])
def test_high_temperatures(nnc, n, k, v, t):
    """Every finite logit near the others, at most a few temperatures apart where logits are as large as the temperature; -infinity, and what lies
    behind a row's end, has no probability however high the temperature is."""
    target, drafts, u, draft = inputs(n, k, v, "f32", t, seed=v, size=1.0)
    for scale in (1.0, 5e37):
        x, y = (target * scale).clamp(-3e38, 3e38), (draft * scale).clamp(-3e38, 3e38)
        check(nnc, x, drafts, u, y, t)
        mask = torch.from_numpy(np.random.default_rng(v).random((n, k + 1, v)) < 0.5)
        mask[:, :k] &= torch.from_numpy(np.arange(v) != drafts[..., None])
        check(nnc, x.masked_fill(mask, -math.inf), drafts, u, None, t)
        check(nnc, x.masked_fill(mask, -math.inf), drafts, u, y.masked_fill(mask[:, :k], -math.inf), t)
        low = x.masked_fill(mask, LOWEST)
        check(nnc, low, drafts, u, None, t)
        low[:, :, v // 2:] = -math.inf
        check(nnc, low, np.minimum(drafts, v // 2 - 1), u, None, t)


@pytest.mark.parametrize("t", [0.0, 1e-45, 1e-3, 0.7, 1.0, 1.3, 1e30, 1e37])
@pytest.mark.parametrize("v,ids", [(5003, 900), (151936, 40000)])
def test_chunks_of_nothing_but_the_lowest_number(nnc, v, ids, t):
    """Everything from some id on masked by the type's lowest number, to the end of a row, alone and mixed with -infinity."""
    target, drafts, u, draft = inputs(6, 2, v, "f32", t if t > 0.5 else 1.0, seed=v)
    target[..., ids:], draft[..., ids:] = LOWEST, LOWEST
    target[3:, :, v - 40:], draft[3:, :, ids + 1024:ids + 4000] = -math.inf, -math.inf
    drafts = np.minimum(drafts, ids - 1)
    if 0 < t < 0.5:                                                       # (what such a temperature leaves: the largest)
        drafts = pu.f64(draft).argmax(-1).astype(np.int32)
    check(nnc, target, drafts, u, draft, t)
    check(nnc, target, drafts, u, None, t)
    check(nnc, target[:, 2:], drafts[:, :0], u[:, 2:], None, t)


@pytest.mark.parametrize("t", [0.0, 1e-45, 1.0, 1e37])
@pytest.mark.parametrize("v", [60, 1024, 5003])
def test_rows_of_nothing_but_the_lowest_number(nnc, v, t):
    """The lowest number is a logit like others: where there is no larger one it has all the probability, in equal parts."""
    x = torch.full((5, 1, v), LOWEST)
    x[1, :, ::2] = -math.inf
    x[2, :, :v // 2] = -math.inf
    x[3, :, 1:] = -math.inf
    x[4, :, v // 3] = LOWEST * (1 - 2.0 ** -23)
    u = np.array([[0.3], [0.51], [0.77], [0.9], [0.2]], np.float32)
    want = check(nnc, x, np.zeros((5, 0), np.int32), u, None, t)
    assert want[0][3, 0] == 0 and (t > 1 or want[0][4, 0] == v // 3)


def test_probabilities_below_those_of_a_random_number(nnc):
    """Drafts whose probabilities lie below 2^-400 of the best token's are compared like others, down to the end of 64 bits; what lies below
    that, as tokens do that a finite mask forbids, is not kept, not even by a random number of zero."""
    v = 3000
    x = torch.zeros((8, 2, v))
    y = torch.zeros((8, 1, v))
    x[..., 7], y[..., 7] = 50.0, 50.0
    far = [(-300.0, -600.0), (-600.0, -300.0), (-400.0, -400.5), (-400.5, -400.0), (-500.0, -499.0), (-1e9, -1e9), (LOWEST, LOWEST), (-2000.0, -3000.0)]
    for i, (p, q) in enumerate(far):
        x[i, :, 99], y[i, :, 99] = p, q
    drafts = np.full((8, 1), 99, np.int32)
    kept = {0.9: [1, 0, 1, 0, 0, 0, 0, 0], 0.5: [1, 0, 1, 1, 0, 0, 0, 0], 0.0: [1, 1, 1, 1, 1, 0, 0, 0]}
    for u0, accepted in kept.items():
        u = np.array([[u0, 0.5]] * 8, np.float32)
        want = check(nnc, x, drafts, u, y, 1.0)
        assert want[1].tolist() == accepted
    # what is left of p behind q is next to nothing, or nothing, where they agree on all that counts
    x[:, :, 5], y[:, :, 5] = -400.0, -700.0
    u = np.array([[0.999, 0.5]] * 8, np.float32)
    got = nnc.draft_verify(x.to(DEV), ints(drafts), torch.from_numpy(u).to(DEV), y.to(DEV))
    want = su.verify(pu.f64(x), drafts, u.astype(np.float64), pu.f64(y), None, [1.0] * 8)
    assert np.array_equal(got[0].cpu().numpy(), want[0])
    u[:, 1] = 0.0                                                          # a mask is never what is picked behind a rejected draft
    x[:, :, :4], y[:, :, :4] = -1e9, -1e9
    got = nnc.draft_verify(x.to(DEV), ints(drafts), torch.from_numpy(u).to(DEV), y.to(DEV))
    want = su.verify(pu.f64(x), drafts, u.astype(np.float64), pu.f64(y), None, [1.0] * 8)
    lost = want[1] == 0
    assert np.array_equal(got[0].cpu().numpy()[lost], want[0][lost]) and (want[0][lost, 0] >= 4).all() and np.array_equal(got[1].cpu().numpy(), want[1])
    # ... but of p itself it is the first number of all, e^(-1e9 - 50) / sum > 0, where the random number is zero (in 64 bits that is a zero, as the definition here has it)
    assert got[0][~torch.from_numpy(lost).to(DEV)].tolist() == [[99, 0]] * int((~lost).sum())
