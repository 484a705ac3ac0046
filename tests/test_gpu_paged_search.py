"""Searches on pages in parts: what one call leaves is what the next one goes on from."""
import numpy as np
import pytest
import torch

import page_util as pu
from parity_util import SMALL_BF16
from test_gpu_paged_model import begin

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def nnc():
    from paper_2512_21571_amd import binding
    binding.lib()
    return binding


@pytest.mark.parametrize("groups,width", [(1, 4), (3, 5)])
def test_ended_beams_stay_ended_without_an_end_token(nnc, groups, width):
    """The beams of a search with an end token go on without one, a step at a time, against the definition: those that have ended keep
    their score and repeat their token, the others go on past a token that no longer ends anything."""
    prompt, steps, shape = 21, 6, SMALL_BF16
    blob, m, pages, tables, logits, lens = begin(nnc, shape, groups, width, prompt, steps + 1, torch.bfloat16)
    _, m2, pages2, tables2, _, lens2 = begin(nnc, shape, groups, width, prompt, steps + 1, torch.bfloat16, blob)
    eos = int(logits[0].float().argsort(descending=True)[1])                 # what the second-best continuation of the prompt begins with
    tok, par, sc, fin = m.decode_beam(pages, tables, lens, 1, first_logits=logits, width=width, eos=eos)
    pages2.reorder(tables2, tables2, lens2, par[-1])
    assert fin.any() and not fin.all()
    seen = 0
    for _ in range(steps):
        last, was = tok[-1].clone(), fin.clone()
        tok, par, sc2, fin = m.decode_beam(pages, tables, lens, 1, tokens=last, scores=sc, finished=was)
        lg, _ = m2.decode_step_paged(pages2, tables2, lens2, last.reshape(-1))
        pages2.reorder(tables2, tables2, lens2, par[-1])
        want = pu.select(pu.f64(lg.unflatten(0, (groups, width))), pu.f64(sc), was.cpu().numpy(), eos)
        assert np.array_equal(tok[0].cpu().numpy(), want[0]) and np.array_equal(par[0].cpu().numpy(), want[1])
        assert np.allclose(pu.f64(sc2), want[2], rtol=2.0 ** -23, atol=2.0 ** -20)
        parent = par[0].long()
        assert torch.equal(fin, was.gather(1, parent))                       # nothing ends, nothing comes back to life
        assert torch.equal(tok[0][fin], last.gather(1, parent)[fin]) and torch.equal(sc2[fin], sc.gather(1, parent)[fin])
        seen += int(fin.sum())
        sc = sc2
    assert seen
    assert torch.equal(tables, tables2) and torch.equal(lens, lens2)
