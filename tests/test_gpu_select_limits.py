"""The beam selection where its contract has an edge: failed beams with forbidden tokens."""
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
