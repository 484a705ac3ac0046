"""Verification of drafted tokens against the definition in 64 bits."""
import math

import numpy as np
import pytest
import torch

import page_util as pu
import share_util as su
from share_util import DEV, ints

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def nnc():
    from paper_2512_21571_amd import binding
    binding.lib()
    return binding


def inputs(n, k, v, rows, seed=1, agree=0.5, size=2.5):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    draft = (torch.randn((n, k, v), generator=gen, device=DEV) * size).to(pu.ROWS[rows])
    target = torch.randn((n, k + 1, v), generator=gen, device=DEV) * agree
    target[:, :k] += draft.float()
    drafts = torch.randint(0, v, (n, k), generator=gen, device=DEV)
    if k:
        noise = -torch.log(-torch.log(torch.rand((n, k, v), generator=gen, device=DEV).clamp(1e-6, 1 - 1e-6)))
        drafts = (draft.float() + noise).argmax(-1)
    return target.to(pu.ROWS[rows]), drafts.int(), torch.rand((n, k + 1), generator=gen, device=DEV), draft


def check(nnc, logits, drafts, uniforms, draft_logits=None, counts=None, temperature=1.0):
    got = nnc.draft_verify(logits, drafts, uniforms, draft_logits, counts=counts, temperature=temperature)
    n = logits.shape[0]
    heat = temperature.cpu().numpy() if isinstance(temperature, torch.Tensor) else np.full(n, np.float32(temperature))
    want = su.verify(pu.f64(logits), drafts.cpu().numpy(), pu.f64(uniforms), None if draft_logits is None else pu.f64(draft_logits),
                     None if counts is None else counts.cpu().numpy(), heat)
    # Exponentials are good to 2^-42 and sums add no more than a few 2^-53, so a quotient of two is within 2^-40; no decision of these inputs is that close.
    assert want[2] > 2.0 ** -40, want[2]
    assert np.array_equal(got[0].cpu().numpy(), want[0]) and np.array_equal(got[1].cpu().numpy(), want[1])
    return got


@pytest.mark.parametrize("rows", list(pu.ROWS))
@pytest.mark.parametrize("n,k,v", [(1, 1, 2), (3, 4, 17), (5, 2, 1023), (2, 5, 1024), (4, 3, 1025), (2, 7, 16385), (3, 4, 151936), (1, 2, 300001), (2, 70, 50)])
def test_verify(nnc, rows, n, k, v):
    target, drafts, u, draft = inputs(n, k, v, rows, seed=v)
    for t in (1.0, 0.6, 0.0, 1.7):
        check(nnc, target, drafts, u, draft, temperature=t)
        check(nnc, target, drafts, u, None, temperature=t)
    counts = ints(np.random.default_rng(v).integers(0, k + 1, n))
    heat = torch.tensor([0.0, 0.7, 1.0, 2.5, 1e-3], device=DEV)[torch.arange(n, device=DEV) % 5].contiguous()
    check(nnc, target, drafts, u, draft, counts, heat)
    check(nnc, target, drafts, u, None, counts, heat)
    best = target[:, :k].argmax(-1).int()
    check(nnc, target, best, u, None, counts, heat)                       # drafts that greedy sequences keep
    check(nnc, target, best, u, draft, None, 0.0)


@pytest.mark.parametrize("rows", list(pu.ROWS))
@pytest.mark.parametrize("v", [1, 5, 2000, 151936])
def test_sampling_without_drafts(nnc, rows, v):
    """k = 0: one token out of the target's distribution, for random numbers over all of [0, 1)."""
    gen = torch.Generator(device=DEV).manual_seed(v)
    n = 40
    logits = (torch.randn((1, 1, v), generator=gen, device=DEV) * 2).to(pu.ROWS[rows]).expand(n, 1, v).contiguous()
    u = (torch.arange(n, device=DEV) / n + 0.003)[:, None].contiguous()
    u[0], u[-1] = 0.0, 1 - 2.0 ** -24
    none = torch.empty((n, 0), dtype=torch.int32, device=DEV)
    got = nnc.draft_verify(logits, none, u)
    assert (got[1] == 0).all() and (got[0][1:] >= got[0][:-1]).all()       # the inverse of a rising function
    x = pu.f64(logits[0, 0])
    sums = np.cumsum(su.softmax(x, 1.0))
    want = np.searchsorted(sums, pu.f64(u)[:, 0] * sums[-1], side="right")
    assert np.array_equal(got[0][:, 0].cpu().numpy(), want)


def test_the_tokens_are_the_targets(nnc):
    """Drafts drawn from q and verified are distributed as p: 200000 sequences over 6 tokens; a frequency of p = 0.2 or so is off by
    sqrt(p (1 - p) / 200000) = 0.0009, and the bound is six of these."""
    rng = np.random.default_rng(5)
    n, v = 20000, 6
    p, q = rng.dirichlet(np.ones(v)), rng.dirichlet(np.ones(v))
    seen = np.zeros(v)
    logits = torch.from_numpy(np.log(p)).float().to(DEV).expand(n, 2, v).contiguous()
    draft = torch.from_numpy(np.log(q)).float().to(DEV).expand(n, 1, v).contiguous()
    for seed in range(10):
        r = np.random.default_rng(seed)
        drafts = ints(r.choice(v, (n, 1), p=q))
        u = torch.from_numpy(r.random((n, 2)).astype(np.float32)).clamp(max=1 - 2.0 ** -24).to(DEV)
        tokens, accepted = nnc.draft_verify(logits, drafts, u, draft)
        seen += np.bincount(tokens[:, 0].cpu().numpy(), minlength=v)
    f = seen / (10 * n)
    assert (np.abs(f - p) <= 6 * np.sqrt(p * (1 - p) / (10 * n))).all()


@pytest.mark.parametrize("rows", list(pu.ROWS))
@pytest.mark.parametrize("v", [40, 5003])
def test_forbidden_tokens_and_far_logits(nnc, rows, v):
    """-infinity in the target (never chosen, a draft of it is not kept), in the draft; logits far from zero; the type's lowest value."""
    target, drafts, u, draft = inputs(6, 3, v, rows, seed=v, agree=1.0)
    mask = torch.rand(target.shape, generator=torch.Generator(device=DEV).manual_seed(1), device=DEV) < 0.6
    mask[..., 0] = False
    t = target.masked_fill(mask, -math.inf)
    got = check(nnc, t, drafts, u, draft)
    check(nnc, t, drafts, u, None)
    for i in range(6):
        for j in range(int(got[1][i]) + 1):
            assert t[i, j, int(got[0][i, j])] > -math.inf
    d = draft.masked_fill(mask[:, :3] & (torch.arange(v, device=DEV) != drafts[..., None]), -math.inf)
    check(nnc, target, drafts, u, d)
    low = torch.where(mask, torch.finfo(target.dtype).min, target)
    check(nnc, low, drafts, u, draft)
    if rows != "f16":
        for offset in (3e4, -2.0 ** 100):
            check(nnc, ((target.float() / 8).clamp(-1, 1) * offset).to(target.dtype), drafts, u, draft, temperature=abs(offset) / 4)


@pytest.mark.parametrize("top", [3.0, -7.5, 0.0, 1e-40, 3.4e38, -3.4e38, 65504.0])
def test_temperatures_so_low_that_only_equals_are_left(nnc, top):
    """Three equal largest logits in three chunks share the probability; the next smaller number has next to none, however near it
    is (but e^-290 and less is more than u = 0 asks for, so that the first token is picked there)."""
    top = np.float32(top)
    x = np.full(5000, np.nextafter(top, np.float32(-np.inf)), np.float32)
    x[1000:2000] = np.float32(-3.4028235e38)
    x[[70, 2500, 4999]] = top
    logits = torch.from_numpy(x).to(DEV).expand(6, 1, 5000).contiguous()
    u = torch.tensor([0.0, 0.32, 0.35, 0.65, 0.68, 1 - 2.0 ** -24], device=DEV)[:, None].contiguous()
    none = torch.empty((6, 0), dtype=torch.int32, device=DEV)
    step = float(top) - float(np.nextafter(top, np.float32(-np.inf)))
    for t in (step / 300, step / 1e6, 1e-45):
        if 0 < np.float32(t) and step / float(np.float32(t)) > 290:       # e^-290 of 5000 others: nothing beside three ones
            assert nnc.draft_verify(logits, none, u, temperature=float(np.float32(t)))[0][:, 0].tolist() == [0, 70, 2500, 2500, 4999, 4999], t


def test_equal_distributions_and_edges_of_the_random_numbers(nnc):
    """p = q: every draft is kept, whatever u; u = 0 keeps whatever has any probability; equal logits; a residual of nothing."""
    target, drafts, u, draft = inputs(4, 3, 777, "f32")
    same = target.clone()
    same[:, :3] = draft
    u[:, :3] = 1 - 2.0 ** -24
    assert nnc.draft_verify(same, drafts, u, draft)[1].tolist() == [3] * 4
    u[:, :3] = 0
    assert nnc.draft_verify(target, drafts, u, draft)[1].tolist() == [3] * 4
    flat = torch.zeros((2, 3, 100), device=DEV)
    u = torch.tensor([[0.5, 0.5, 0.995], [0.0, 0.02, 0.0]], device=DEV)
    drafts = ints([[3, 4], [5, 6]])
    got = nnc.draft_verify(flat, drafts, u, flat[:, :2].contiguous())
    assert got[0].tolist() == [[3, 4, 99], [5, 6, 0]]
    assert nnc.draft_verify(flat, drafts, u)[0].tolist() == [[99, -1, -1], [5, 0, -1]]
    assert nnc.draft_verify(flat, drafts, u, temperature=0.0)[0].tolist() == [[0, -1, -1], [0, -1, -1]]     # ties: the lowest index
    one = torch.full((1, 2, 9), -math.inf, device=DEV)                       # the target has one token, and the draft is another
    one[..., 4] = 1.0
    assert nnc.draft_verify(one, ints([[4]]), torch.tensor([[0.999, 0.5]], device=DEV))[0].tolist() == [[4, 4]]
    assert nnc.draft_verify(one, ints([[2]]), torch.tensor([[0.0, 0.5]], device=DEV))[0].tolist() == [[4, -1]]


def test_failures_show_and_what_is_not_looked_at_does_not(nnc):
    target, drafts, u, draft = inputs(8, 3, 3000, "f32", agree=0.0)
    target[:, :3] = draft
    u[:, :3] = 0.25
    clean = nnc.draft_verify(target, drafts, u, draft)
    assert clean[1].tolist() == [3] * 8
    target[0, 2, 2999] = math.nan
    target[1, 0, 5] = math.inf
    target[2, 1] = -math.inf
    draft[3, 1, 17] = math.nan
    drafts[4, 0], drafts[5, 2] = 3000, -1
    u[6, 1] = math.nan
    u[7, 3] = math.nan
    tokens, accepted = nnc.draft_verify(target, drafts, u, draft)
    assert accepted.tolist() == [2, 0, 1, 1, 0, 2, 1, 3]
    for i, a in enumerate(accepted.tolist()):
        assert tokens[i].tolist() == drafts[i, :a].tolist() + [-1] * (4 - a)
    # rows behind a rejection or behind the count are not looked at
    target, drafts, u, draft = inputs(3, 3, 3000, "f32", agree=0.0)
    target[:, :3] = draft
    target[:, 2:], draft[:, 2] = math.nan, math.nan
    counts = ints([1, 2, 0])
    u[:, :3] = 0.25
    u[1, 1] = 1.0
    target[1, 1, int(drafts[1, 1])] -= 5
    got = nnc.draft_verify(target, drafts, u, draft, counts=counts)
    want = su.verify(pu.f64(target), drafts.cpu().numpy(), pu.f64(u), pu.f64(draft), [1, 2, 0], [1.0] * 3)
    assert np.array_equal(got[0].cpu().numpy(), want[0]) and got[1].tolist() == [1, 1, 0] and (got[0][:, 0] >= 0).all()
    # counts and temperatures out of range
    got = nnc.draft_verify(target, drafts, u, draft, counts=ints([-1, 4, 1]), temperature=torch.tensor([1.0, 1.0, -1.0], device=DEV))
    assert (got[0] == -1).all() and got[1].tolist() == [0, 0, 0]
    got = nnc.draft_verify(target, drafts, u, draft, counts=ints([1, 1, 1]), temperature=torch.tensor([math.nan, math.inf, 1.0], device=DEV))
    assert (got[0][:2] == -1).all() and got[1].tolist()[:2] == [0, 0] and got[0][2, 0] == drafts[2, 0]


def test_strides_streams_and_workspaces(nnc):
    """Rows at every alignment, more than 2^32 bytes apart; the same call the same tokens; on a stream of the caller's."""
    for rows in pu.ROWS:
        target, drafts, u, draft = inputs(2, 3, 4099, rows)
        wide = torch.zeros((8, 4107), dtype=target.dtype, device=DEV)
        wide[:, 3:4102] = target.flatten(0, 1)
        t = wide[:, 3:4102].unflatten(0, (2, 4))
        a, b = nnc.draft_verify(t, drafts, u, draft), nnc.draft_verify(target, drafts, u, draft)
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    step = 1_100_000_007
    base = torch.empty(3 * step + 6000, device=DEV)
    far = base.as_strided((2, 2, 5000), (2 * step, step, 1))
    target, drafts, u, draft = inputs(2, 1, 5000, "f32")
    far.copy_(target)
    want = nnc.draft_verify(target, drafts, u, draft)
    ws = torch.empty(1 << 20, dtype=torch.uint8, device=DEV)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = nnc.draft_verify(far, drafts, u, draft, workspace=ws)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    with pytest.raises(nnc.NncError):
        nnc.draft_verify(target, drafts, u, draft, workspace=ws[:64])
    for change in (dict(drafts=drafts.long()), dict(uniforms=u[:, :1]), dict(draft_logits=draft.half()), dict(draft_logits=target), dict(counts=torch.zeros(3, dtype=torch.int32, device=DEV)),
                   dict(temperature=-1.0), dict(temperature=torch.ones(3, device=DEV)), dict(logits=target[..., ::2]), dict(drafts=drafts.cpu())):
        with pytest.raises(nnc.NncError):
            nnc.draft_verify(**{**dict(logits=target, drafts=drafts, uniforms=u, draft_logits=draft), **change})
    empty = nnc.draft_verify(target[:0], drafts[:0], u[:0], draft[:0])
    assert empty[0].shape == (0, 2) and empty[1].shape == (0,)


def test_in_a_graph(nnc):
    target, drafts, u, draft = inputs(3, 4, 9001, "bf16")
    for _ in range(2):
        nnc.draft_verify(target, drafts, u, draft)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = nnc.draft_verify(target, drafts, u, draft)
    for seed in range(4):
        for a, b in zip((target, drafts, u, draft), inputs(3, 4, 9001, "bf16", seed=seed)):
            a.copy_(b)
        g.replay()
        got = [x.clone() for x in out]
        want = nnc.draft_verify(target, drafts, u, draft)
        torch.cuda.synchronize()
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
