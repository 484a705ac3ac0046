"""A model's pass over as many drafts as it takes, and over contexts that several workgroups share, against its steps one by one."""
import numpy as np
import pytest
import torch

from parity_util import SMALL_BF16, SMALL_F16, SMALL_F32, SMALL_G4
from test_gpu_paged_model import DEV, POOL, nnc, setup  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("shape", [SMALL_BF16, SMALL_G4, SMALL_F16, SMALL_F32], ids=lambda s: s.name)
@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("lens,k", [([700], 20), ([50], 20), ([640, 33], 9), ([5, 900, 129], 6), ([300, 20, 7, 511, 64, 1, 90], 2), ([20] * 21, 0)])
def test_wide_passes_and_long_contexts(nnc, shape, eight, lens, k):  # noqa: F811
    """The bounds of test_one_pass_equals_steps_one_by_one: 4e-3 of either side against the oracle, of an 8-bit cache a hundredth of the logits' span."""
    _, m, pages, tables, first = setup(nnc, shape, lens, torch.int8 if eight else POOL[shape.dtype], steps=k + 1, max_seq=max(lens) + k + 8)
    rng = np.random.default_rng(3)
    tokens = torch.from_numpy(np.concatenate([np.array(first)[:, None], rng.integers(0, shape.vocab, (len(lens), k))], 1).astype(np.int32)).to(DEV)
    ln = torch.tensor(lens, dtype=torch.int32, device=DEV)
    want = []
    for j in range(k + 1):
        want.append(m.decode_step_paged(pages, tables, ln, tokens[:, j].contiguous())[0])
    want = torch.stack(want, 1)
    start = torch.tensor(lens, dtype=torch.int32, device=DEV)
    for max_len in (0, max(lens)):
        got, nxt = m.decode_step_drafts(pages, tables, start, tokens, max_len=max_len, want_next=True)
        bound = 8e-3 if not eight else 0.02 * float(want.max() - want.min())
        assert float((got - want).abs().max()) <= bound
        assert torch.equal(nxt, got.argmax(-1).int())
