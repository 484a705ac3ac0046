"""A model on pages where its contexts are long enough for the attention to be split, with as many sequences as a step has columns,
and the rows that a step itself quantises."""
import numpy as np
import pytest
import torch

import page_util as pu
import synth
from parity_util import SMALL_BF16, SMALL_F16, SMALL_F32, SMALL_G4
from test_gpu_pages import same_bits
from test_gpu_paged_model import POOL, SMALL_W8

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
MAX_SEQ = 4096


@pytest.fixture(scope="module")
def nnc():
    from paper_2512_21571_amd import binding
    binding.lib()
    return binding


def setup(nnc, shape, lens, dtype, tokens, steps):
    """A model with a prompt in a slot for each length, and pages of another order with the same rows."""
    m = nnc.Model(shape, synth.make_blob(shape, weight_std=0.05), len(lens), MAX_SEQ)
    per = -(-(max(lens) + steps) // tokens)
    pages = nnc.Pages.empty(shape.n_layers, len(lens) * per, tokens, shape.n_kv_heads, 128, dtype, DEV)
    tables = torch.from_numpy(np.random.default_rng(1).permutation(pages.n_pages).reshape(len(lens), per).astype(np.int32)).to(DEV)
    first = []
    for s, n in enumerate(lens):
        first.append(int(m.prefill(s, synth.tokens(n, shape.vocab, stream=s))[1].item()))
        m.pages_store(pages, tables, s, s)
    return m, pages, tables, first


def some_lengths(n):
    return [3000, 300, 1, 257, 256, 2048, 1023, 700, 64, 511, 2999, 128, 1500, 20, 900, 2047, 333, 260, 1024, 5, 2500][:n]


@pytest.mark.parametrize("shape,n", [(SMALL_BF16, 1), (SMALL_BF16, 7), (SMALL_BF16, 16), (SMALL_BF16, 21), (SMALL_G4, 6), (SMALL_G4, 12), (SMALL_F16, 1),
                                     (SMALL_F16, 16), (SMALL_F32, 1), (SMALL_F32, 7), (SMALL_W8, 7), (SMALL_W8, 16)], ids=lambda x: str(getattr(x, "name", x)))
def test_long_contexts_on_pages_equal_slots(nnc, shape, n):
    """Up to 3000 positions (24 splits of one sequence), and every number of 16-bit pieces that a step's operands take.  The same tokens go
    into both; the logits agree to the bound that the small models keep against the oracle (4e-3)."""
    lens, steps = some_lengths(n), 3
    m, pages, tables, first = setup(nnc, shape, lens, POOL[shape.dtype], 16, steps)
    ln = torch.tensor(lens, dtype=torch.int32, device=DEV)
    tok = torch.tensor(first, dtype=torch.int32, device=DEV)
    for step in range(steps):
        want, nxt = m.decode_step(list(range(n)), tok.tolist())
        got, _ = m.decode_step_paged(pages, tables, ln, tok, max_len=max(lens) + step if step == 1 else 0)
        assert float((got - want).abs().max()) <= 4e-3
        tok = nxt.clone()
    m.synchronize()
    assert ln.tolist() == [x + steps for x in lens]


def test_one_sequence_with_and_without_neighbours(nnc):
    """A sequence's logits do not depend on who else is in the step, but for the order of sums: alone, the attention is split more
    finely and operands are in three pieces, among sixteen in two (2^-17)."""
    lens = some_lengths(16)
    m, pages, tables, first = setup(nnc, SMALL_BF16, lens, torch.bfloat16, 32, 1)
    ln = torch.tensor(lens, dtype=torch.int32, device=DEV)
    tok = torch.tensor(first, dtype=torch.int32, device=DEV)
    alone = [m.decode_step_paged(pages, tables[i:i + 1].contiguous(), ln[i:i + 1].clone(), tok[i:i + 1].clone())[0] for i in (0, 3, 5)]
    got, _ = m.decode_step_paged(pages, tables, ln, tok)
    for i, a in zip((0, 3, 5), alone):
        assert float((got[i] - a[0]).abs().max()) <= 4e-3


def test_a_search_over_a_long_prompt_is_its_operators_one_by_one(nnc):
    prompt, width, steps, tokens = 900, 6, 5, 32
    shape, full = SMALL_BF16, 900 // 32
    runs = []
    for _ in range(2):
        m = nnc.Model(shape, synth.make_blob(shape, weight_std=0.05), 1, 1024)
        per = -(-(prompt + steps) // tokens)
        pages = nnc.Pages.empty(shape.n_layers, full + width * (per - full), tokens, shape.n_kv_heads, 128, torch.float8_e4m3fn, DEV)
        ids = np.random.default_rng(2).permutation(pages.n_pages).astype(np.int32)
        t = np.zeros((width, per), np.int32)
        t[:, :full], t[:, full:] = ids[None, :full], ids[full:].reshape(width, per - full)
        tables = torch.from_numpy(t).to(DEV)
        logits, _ = m.prefill(0, synth.tokens(prompt, shape.vocab, stream=3))
        m.pages_store(pages, tables, 0, 0)
        runs.append((m, pages, tables, logits[None], torch.full((width,), prompt, dtype=torch.int32, device=DEV)))
    m, pages, tables, logits, lens = runs[0]
    toks, pars, scores, _ = m.decode_beam(pages, tables, lens, steps, first_logits=logits, width=width)
    m, pages2, tables2, logits, lens2 = runs[1]
    sc = torch.full((1, width), -torch.inf, device=DEV)
    sc[:, 0] = 0
    lg = logits[:, None].expand(1, width, shape.vocab).contiguous()
    for step in range(steps):
        tok, par, sc, _ = nnc.beam_select(lg, sc)
        pages2.reorder(tables2, tables2, lens2, par)
        assert torch.equal(tok, toks[step]) and torch.equal(par, pars[step])
        if step + 1 < steps:
            lg = m.decode_step_paged(pages2, tables2, lens2, tok.reshape(-1))[0][None]
    assert torch.equal(sc, scores) and torch.equal(tables, tables2) and torch.equal(lens, lens2)


@pytest.mark.parametrize("shape", [SMALL_BF16, SMALL_G4, SMALL_F32], ids=lambda s: s.name)
@pytest.mark.parametrize("store", ["i8", "e4m3", "bf16", "f16"])
def test_a_step_stores_what_append_stores(nnc, shape, store):
    """The first layer's new rows (they depend on the token and its position alone) as an fp32 pool holds them, appended to a pool of
    the format: the same bytes and scales as a step's own."""
    n = 16
    lens = some_lengths(n)
    rows = []
    for dtype in (torch.float32, pu.STORES[store]):
        m, pages, tables, first = setup(nnc, shape, lens, dtype, 24, 1)
        ln = torch.tensor(lens, dtype=torch.int32, device=DEV)
        m.decode_step_paged(pages, tables, ln, torch.tensor([(7 * i + 1) % shape.vocab for i in range(n)], dtype=torch.int32, device=DEV))
        rows.append((pages, tables))
    (exact, t0), (pages, t1) = rows
    at = torch.tensor(lens, dtype=torch.int32, device=DEV)
    seq = torch.arange(n, dtype=torch.int32, device=DEV)
    k, v = exact.read(0, t0, seq, at)
    other = nnc.Pages.empty(1, n, 24, shape.n_kv_heads, 128, pu.STORES[store], DEV)
    own = torch.arange(n, dtype=torch.int32, device=DEV)[:, None]
    other.append(0, k, v, own, seq, torch.zeros_like(seq))
    page, row = t1[seq.long(), (at // 24).long()].long(), (at % 24).long()
    for a, b in ((pages.k, other.k), (pages.v, other.v), (pages.k_scale, other.k_scale), (pages.v_scale, other.v_scale)):
        if a is None:
            continue
        a, b = (x.view(torch.uint8) if x.dtype == torch.float8_e4m3fn else x for x in (a, b))
        assert same_bits(a[0, page, :, row].contiguous(), b[0, :, :, 0].contiguous())
