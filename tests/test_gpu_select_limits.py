"""The beam selection where its contract has an edge: failed beams with forbidden tokens, the error of the log-sum;
and wide searches over rows of more chunks than beams, where a wave looks into the best chunks of one beam or of two."""
import math

import numpy as np
import pytest
import torch

import page_util as pu
from test_gpu_pages import check_select

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def nnc():
    from paper_2512_21571_amd import binding
    binding.lib()
    return binding


@pytest.mark.parametrize("rows", list(pu.ROWS))
@pytest.mark.parametrize("v", [50, 5000, 40000])
@pytest.mark.parametrize("failure", [math.nan, math.inf])
def test_forbidden_tokens_of_a_failed_beam_stay_forbidden(nnc, rows, v, failure):
    """A beam with a NaN or a +infinity among its logits: every token of it that is not forbidden has the score NaN and goes first, the
    larger logit before the smaller one; the forbidden ones keep -infinity and come after every number."""
    w, top = 6, v // 3
    x = torch.randn((1, w, v), generator=torch.Generator(device=DEV).manual_seed(v), device=DEV).to(pu.ROWS[rows])
    x[0, 2] = -math.inf
    x[0, 2, top], x[0, 2, 7], x[0, 2, 9] = failure, 1.0, 2.0
    scores = torch.full((1, w), -1.0, device=DEV)
    tokens, parents, out, _ = nnc.beam_select(x, scores)
    assert parents[0, :3].tolist() == [2] * 3 and tokens[0, :3].tolist() == [top, 9, 7] and out[0, :3].isnan().all()
    assert 2 not in parents[0, 3:].tolist() and torch.isfinite(out[0, 3:]).all()
    # where nothing else is left (the other beams are not in use), they are chosen, in order
    scores[:] = -math.inf
    scores[0, 2] = -1.0
    tokens, parents, out, _ = nnc.beam_select(x, scores)
    assert tokens[0, :3].tolist() == [top, 9, 7] and out[0, :3].isnan().all() and (out[0, 3:] == -math.inf).all()
    assert parents[0, 3:].tolist() == [0] * 3 and tokens[0, 3:].tolist() == [0, 1, 2]


@pytest.mark.parametrize("rows", list(pu.ROWS))
@pytest.mark.parametrize("v", [40, 1024, 33000, 151936, 600000])
@pytest.mark.parametrize("scale,offset", [(0.01, 0.0), (2.5, 0.0), (6.0, 0.0), (2.5, 800.0)])
def test_the_log_sum_is_good_to_fp32(nnc, rows, v, scale, offset):
    """Seen in scores next to zero (a beam that begins at its log-sum less its best logit), whose own rounding is below 2^-40.  An
    exponential is off by 2^-23, its exponent (17 in base 2 at most where weight is) by 2^-24 of itself in the scan and again
    when chunks are joined, 24 roundings of sums: 52 x 2^-24 and less in all, below 2^-18."""
    gen = torch.Generator(device=DEV).manual_seed(v)
    x = (torch.randn((16, 1, v), generator=gen, device=DEV) * scale + offset).to(pu.ROWS[rows])
    d = x.double()
    top = d.amax(-1)
    lse = top + torch.log(torch.exp(d - top[..., None]).sum(-1))
    start = (lse - top).float()
    got = nnc.beam_select(x, start)
    assert torch.equal(got[0], (x == x.amax(-1, keepdim=True)).int().argmax(-1).int())
    assert float((got[2].double() - (start.double() + (top - lse))).abs().max()) <= 2.0 ** -18


def test_equal_rows_have_equal_log_sums(nnc):
    """Whatever the alignment of a row, so that a tie of two beams is a tie: the lower beam first."""
    for v in (999, 20011, 151936):
        gen = torch.Generator(device=DEV).manual_seed(v)
        wide = torch.zeros((8, v + 1), device=DEV, dtype=torch.bfloat16)
        wide[:, :v] = torch.randn(v, generator=gen, device=DEV)
        tokens, parents, out, _ = nnc.beam_select(wide[:, :v][None], torch.full((1, 8), -3.0, device=DEV))
        assert parents[0].tolist() == list(range(8)) and len(set(out[0].tolist())) == 1 and len(set(tokens[0].tolist())) == 1


WIDE = [(2, 12, 151936), (1, 16, 33000), (3, 9, 9217), (1, 17, 40000), (1, 24, 300001), (1, 32, 151936)]


@pytest.mark.parametrize("rows", list(pu.ROWS))
@pytest.mark.parametrize("g,w,v", WIDE)
def test_wide_searches(nnc, rows, g, w, v):
    gen = torch.Generator(device=DEV).manual_seed(v)
    logits = (torch.randn((g * w, v + 3), generator=gen, device=DEV) * 3).to(pu.ROWS[rows])[:, 3:].unflatten(0, (g, w))
    scores = -torch.rand((g, w), generator=gen, device=DEV) * 0.5 - 20      # (close together: every beam has its share of the best)
    check_select(nnc, logits, scores)
    finished = torch.rand((g, w), generator=gen, device=DEV) < 0.3
    check_select(nnc, logits, scores, finished, v // 2)
    check_select(nnc, logits.masked_fill(torch.rand((g, w, v), generator=gen, device=DEV) < 0.7, -math.inf), scores, finished, v // 2)
    scores[:, 1:] = -math.inf                                               # one beam alone has all the continuations
    check_select(nnc, logits, scores)


@pytest.mark.parametrize("rows", list(pu.ROWS))
@pytest.mark.parametrize("g,w,v", [(1, 16, 33000), (1, 17, 40000), (1, 32, 66000)])
def test_wide_searches_where_the_best_are_neighbours_or_equal(nnc, rows, g, w, v):
    """More candidates than a wave collects at once, in both of its beams and in one of them: the bar is raised, or every place looked for."""
    gen = torch.Generator(device=DEV).manual_seed(w)
    scores = -torch.rand((g, w), generator=gen, device=DEV) * 0.01 - 1
    logits = torch.randn((g, w, v), generator=gen, device=DEV)
    down, few = logits.sort(-1, descending=True)[0], (logits * 0.4).round()
    check_select(nnc, down.to(pu.ROWS[rows]), scores)
    check_select(nnc, logits.sort(-1)[0].to(pu.ROWS[rows]), scores)
    check_select(nnc, few.to(pu.ROWS[rows]), scores)
    check_select(nnc, torch.full_like(logits, 1.25).to(pu.ROWS[rows]), scores)
    mixed = logits.clone()
    mixed[:, ::2], mixed[:, 1::3] = few[:, ::2], down[:, 1::3]
    check_select(nnc, mixed.to(pu.ROWS[rows]), scores)
    stripe = logits.clone()                                                 # two large values in every quarter, always in the same lane
    stripe[:, :, 8:v:256] += 20
    stripe[:, :, 9:v:256] += 20
    check_select(nnc, stripe.to(pu.ROWS[rows]), scores)
