"""A model that verifies drafted tokens on pages: its pass over several tokens of a sequence against its steps one by one, and a run of
drafting and verifying against greedy decoding."""
import numpy as np
import pytest
import torch

import synth
from parity_util import SMALL_BF16, SMALL_F16, SMALL_F32, SMALL_G4
from test_gpu_paged_model import POOL, SMALL_W8, setup

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def nnc():
    from paper_2512_21571_amd import binding
    binding.lib()
    return binding


@pytest.mark.parametrize("shape", [SMALL_BF16, SMALL_G4, SMALL_F16, SMALL_F32, SMALL_W8], ids=lambda s: s.name)
@pytest.mark.parametrize("eight", [False, True])
def test_one_pass_equals_steps_one_by_one(nnc, shape, eight):
    """The bound that the steps of the small models keep against the oracle (4e-3), twice: two passes whose batches differ."""
    lens, k = [1, 16, 33, 62], 3
    _, m, pages, tables, first = setup(nnc, shape, lens, torch.int8 if eight else POOL[shape.dtype])
    rng = np.random.default_rng(3)
    tokens = torch.from_numpy(np.concatenate([np.array(first)[:, None], rng.integers(0, shape.vocab, (4, k))], 1).astype(np.int32)).to(DEV)
    ln = torch.tensor(lens, dtype=torch.int32, device=DEV)
    want = []
    for j in range(k + 1):
        want.append(m.decode_step_paged(pages, tables, ln, tokens[:, j].contiguous())[0])
    want = torch.stack(want, 1)
    rows = [pages.read(1, tables, s, n, n=k + 1) for s, n in enumerate(lens)]
    start = torch.tensor(lens, dtype=torch.int32, device=DEV)
    for max_len in (0, 62):
        got, nxt = m.decode_step_drafts(pages, tables, start, tokens, max_len=max_len, want_next=True)
        assert start.tolist() == lens
        span = 1.0 if not eight else float(want.max() - want.min())
        assert float((got - want).abs().max()) <= (8e-3 if not eight else 0.02 * span)
        assert torch.equal(nxt, got.argmax(-1).int())
    for s, n in enumerate(lens):
        back = pages.read(1, tables, s, n, n=k + 1)
        for a, b in zip(rows[s], back):
            top = a.abs().amax(-1, keepdim=True)
            ulp = {torch.bfloat16: 2.0 ** -7, torch.float16: 2.0 ** -10, torch.float32: 2.0 ** -16, torch.int8: 0}[pages.k.dtype]
            assert ((a - b).abs() <= ulp * a.abs().clamp(min=2.0 ** -6) + 1e-3 + (top / 127 * 1.05 if eight else 0)).all()


def test_counts_wrong_tokens_and_lengths(nnc):
    lens = [20, 20, 20, 20, 20]
    _, m, pages, tables, first = setup(nnc, SMALL_BF16, lens, torch.bfloat16)
    tokens = torch.tensor([[f, 5, 6] for f in first], dtype=torch.int32, device=DEV)
    ln = torch.tensor([20, 20, -1, 20, 26], dtype=torch.int32, device=DEV)
    want, _ = m.decode_step_drafts(pages, tables, torch.tensor(lens, dtype=torch.int32, device=DEV), tokens)
    for t in (pages.k, pages.v):
        t.fill_(float("nan"))
    for s in range(5):
        m.pages_store(pages, tables, s, s)
    before = pages.k.view(torch.int16).clone()
    tokens[3, 1] = SMALL_BF16.vocab
    counts = torch.tensor([2, 1, 2, 2, 2], dtype=torch.int32, device=DEV)
    got, _ = m.decode_step_drafts(pages, tables, ln, tokens, counts=counts, max_len=25)
    ok = [[True] * 3, [True, True, False], [False] * 3, [True, False, False], [False] * 3]
    for i in range(5):
        for j in range(3):
            if ok[i][j]:
                assert torch.equal(got[i, j], want[i, j]), (i, j)
            else:
                assert got[i, j].isnan().all(), (i, j)
    changed = {tuple(x) for x in (pages.k.view(torch.int16) != before).any(-1).any(0).any(1).nonzero().tolist()}   # (page, row)
    assert changed == {(int(tables[i, 1]), 4 + j) for i in range(5) for j in range(3) if ok[i][j]}
    for bad in (-1, 3):
        got, _ = m.decode_step_drafts(pages, tables, ln, tokens, counts=torch.full((5,), bad, dtype=torch.int32, device=DEV), max_len=25)
        assert got.isnan().all()
    with pytest.raises(nnc.NncError) as e:
        m.decode_step_drafts(pages, tables, ln, tokens, max_len=30)               # two pages of 16 hold 32
    assert e.value.status == nnc.E_KV_FULL
    for change in (dict(tokens=torch.zeros((5, 5), dtype=torch.int32, device=DEV)), dict(tokens=tokens.long()), dict(tokens=tokens[:4].contiguous()), dict(counts=counts[:3]),
                   dict(lens=ln[:4]), dict(max_len=1 << 32), dict(tokens=tokens[:, :0])):
        with pytest.raises(nnc.NncError) as e:
            m.decode_step_drafts(**{**dict(pages=pages, tables=tables, lens=ln, tokens=tokens), **change})
        assert e.value.status == nnc.E_ARG
    m.synchronize()


@pytest.mark.parametrize("shape", [SMALL_F32, SMALL_BF16], ids=lambda s: s.name)
def test_drafting_and_verifying_gives_the_greedy_tokens(nnc, shape):
    """Three sequences, drafts that are right, partly right and wrong, greedy verification: the tokens of greedy decoding, in fewer passes."""
    lens, k, steps = [20, 5, 33], 4, 24
    _, m, pages, tables, first = setup(nnc, shape, lens, POOL[shape.dtype], steps=steps + k + 2, max_seq=96)
    want, _ = m.decode_greedy([0, 1, 2], first, steps)
    want = np.concatenate([np.array(first)[None], want.cpu().numpy()]).T          # [sequence][token]
    rng = np.random.default_rng(1)
    ln = torch.tensor(lens, dtype=torch.int32, device=DEV)
    out, passes = [[f] for f in first], 0
    while min(len(o) for o in out) < steps:
        tokens = np.zeros((3, k + 1), np.int32)
        for i, o in enumerate(out):
            at = len(o) - 1
            tokens[i] = np.resize(want[i, at:at + k + 1], k + 1)
            wrong = rng.integers(0, k + 1)
            if wrong < k:
                tokens[i, 1 + wrong] = (tokens[i, 1 + wrong] + 1) % shape.vocab
        t = torch.from_numpy(tokens).to(DEV)
        logits, _ = m.decode_step_drafts(pages, tables, ln, t)
        got, accepted = nnc.draft_verify(logits, t[:, 1:].contiguous(), torch.rand((3, k + 1), device=DEV), temperature=0.0)
        ln += accepted + 1
        passes += 1
        for i in range(3):
            out[i] += got[i, :int(accepted[i]) + 1].tolist()
        if max(len(o) for o in out) > steps + 1:
            break
    for i in range(3):
        n = min(len(out[i]), steps + 1)
        assert out[i][:n] == want[i, :n].tolist(), i
    assert passes < steps / 2 + 2


def test_profile_counts_a_sequences_rows_once(nnc):
    lens = [60, 20]
    _, m, pages, tables, first = setup(nnc, SMALL_BF16, lens, torch.bfloat16)
    tokens = torch.tensor([[f, 1, 2] for f in first], dtype=torch.int32, device=DEV)
    m.profile_begin()
    m.decode_step_drafts(pages, tables, torch.tensor(lens, dtype=torch.int32, device=DEV), tokens)
    got = {r["name"]: r for r in m.profile_end()}
    assert got["page_attention"]["bytes"] == 2 * (63 + 23) * 2 * 2 * 256
    assert got["page_attention"]["flops"] == 2 * (61 + 62 + 63 + 21 + 22 + 23) * 4 * 4 * 128
