"""A model that decodes from pages: against its own slots, against the oracle, and a beam search against both."""
import math

import numpy as np
import pytest
import torch

import oracle
import synth
from parity_util import SMALL_BF16, SMALL_F16, SMALL_F32, SMALL_G4, oracle_flags

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
SMALL_W8 = synth.ModelShape("small-w8", hidden=256, n_layers=2, n_q_heads=4, n_kv_heads=2, head_dim=128, ffn=512, vocab=1024, dtype=synth.W8)
POOL = {synth.BF16: torch.bfloat16, synth.F16: torch.float16, synth.F32: torch.float32, synth.W8: torch.bfloat16}


@pytest.fixture(scope="module")
def nnc():
    from paper_2512_21571_amd import binding
    binding.lib()
    return binding


def setup(nnc, shape, lens, dtype, tokens=16, steps=8, max_seq=96):
    """A model with a slot per sequence holding a prompt, and pages with the same rows."""
    blob = synth.make_blob(shape, weight_std=0.05)
    m = nnc.Model(shape, blob, len(lens), max_seq)
    per = -(-(max(lens) + steps) // tokens)
    rng = np.random.default_rng(1)
    pages = nnc.Pages.empty(shape.n_layers, len(lens) * per, tokens, shape.n_kv_heads, 128, dtype, DEV)
    tables = torch.from_numpy(rng.permutation(pages.n_pages).reshape(len(lens), per).astype(np.int32)).to(DEV)
    first = []
    for s, n in enumerate(lens):
        _, nx = m.prefill(s, synth.tokens(n, shape.vocab, stream=s))
        first.append(int(nx.item()))
        m.pages_store(pages, tables, s, s)
    return blob, m, pages, tables, first


@pytest.mark.parametrize("shape", [SMALL_BF16, SMALL_G4, SMALL_F16, SMALL_F32, SMALL_W8], ids=lambda s: s.name)
def test_steps_on_pages_equal_steps_on_slots(nnc, shape):
    """Same cache type: the same rows but for a last bit that rounds the other way, the same logits to the bound the small models
    keep against the oracle (4e-3), the same greedy tokens."""
    lens = [1, 16, 33, 64, 20]
    blob, m, pages, tables, first = setup(nnc, shape, lens, POOL[shape.dtype])
    ln = torch.tensor(lens, dtype=torch.int32, device=DEV)
    tok = torch.tensor(first, dtype=torch.int32, device=DEV)
    for step in range(6):
        want, nxt = m.decode_step(list(range(5)), tok.tolist())
        got, nx2 = m.decode_step_paged(pages, tables, ln, tok, max_len=max(lens) + step if step % 2 else 0)
        assert float((got - want).abs().max()) <= 4e-3
        assert torch.equal(nxt, nx2)
        tok = nxt.clone()
    m.synchronize()
    assert ln.tolist() == [n + 6 for n in lens]
    for s, n in enumerate(lens):
        for which in range(2):
            a = m.kv_read(1, s, which, 0, n + 6).reshape(n + 6, shape.n_kv_heads, 128)
            b = pages.read(1, tables, s, 0, n=n + 6)[which]
            assert torch.equal(a[:n], b[:n])                              # the prompt's rows are the slot's
            ulp = {torch.bfloat16: 2.0 ** -7, torch.float16: 2.0 ** -10, torch.float32: 2.0 ** -16}[pages.k.dtype]
            assert ((a - b).abs() <= ulp * a.abs().clamp(min=2.0 ** -6) + 1e-4).all()


@pytest.mark.parametrize("dtype", [torch.int8, torch.float8_e4m3fn])
def test_steps_on_eight_bit_pages(nnc, dtype):
    """Rows are the quantised rows of the slots (off by half a step), and one step's logits are those of an attention over the rows
    as they read back: a second model whose slots hold exactly these values cannot be made, so the bound on the logits is the
    cache's: a relative error e of every row moves them by no more than a few e of their range."""
    lens = [40, 7]
    blob, m, pages, tables, first = setup(nnc, SMALL_BF16, lens, dtype)
    for s, n in enumerate(lens):
        for layer in range(2):
            back = pages.read(layer, tables, s, 0, n=n)
            for which in range(2):
                a = m.kv_read(layer, s, which, 0, n).reshape(n, 2, 128)
                top = a.abs().amax(-1, keepdim=True)
                tol = top / 254 * 1.0001 if dtype == torch.int8 else (a.abs() * 2.0 ** -4).clamp(min=0) + top / 448 * 2.0 ** -10 * 1.001
                assert ((back[which] - a).abs() <= tol + a.abs() * 2.0 ** -22).all()
    ln = torch.tensor(lens, dtype=torch.int32, device=DEV)
    tok = torch.tensor(first, dtype=torch.int32, device=DEV)
    want, _ = m.decode_step([0, 1], first)
    got, _ = m.decode_step_paged(pages, tables, ln, tok)
    span = float(want.max() - want.min())
    assert float((got - want).abs().max()) <= (0.02 if dtype == torch.int8 else 0.12) * span
    # the new row was quantised inside the step as nnc_page_append quantises: from the slot's bf16 row it differs by half a step and a rounding
    for which in range(2):
        a = m.kv_read(0, 0, which, lens[0], 1).reshape(2, 128)
        b = pages.read(0, tables, 0, lens[0], n=1)[which][0]
        top = a.abs().amax(-1, keepdim=True)
        tol = (top / 254 if dtype == torch.int8 else a.abs() * 2.0 ** -4 + top / 448 * 2.0 ** -10) * 1.02 + a.abs() * 2.0 ** -7
        assert ((b - a).abs() <= tol).all()


def test_wrong_tokens_and_lengths_show(nnc):
    lens = [20, 20, 20, 20]
    blob, m, pages, tables, first = setup(nnc, SMALL_BF16, lens, torch.bfloat16)
    ln = torch.tensor([20, 20, -1, 31], dtype=torch.int32, device=DEV)
    tok = torch.tensor([first[0], 1024, first[2], first[3]], dtype=torch.int32, device=DEV)
    before = pages.k.view(torch.int16).clone()                             # (bits: rows that nothing was stored in may be NaN)
    got, _ = m.decode_step_paged(pages, tables, ln, tok, max_len=25)
    want, _ = m.decode_step([0], [first[0]])
    assert float((got[0] - want[0]).abs().max()) <= 4e-3
    assert got[1:].isnan().all()
    assert ln.tolist() == [21, 20, -1, 31]
    changed = (pages.k.view(torch.int16) != before).any(-1).any(0).any(1).nonzero().tolist()   # (page, row) pairs
    assert changed == [[int(tables[0, 1]), 4]]
    with pytest.raises(nnc.NncError) as e:
        m.decode_step_paged(pages, tables, ln, tok, max_len=32)               # two pages of 16 hold 32
    assert e.value.status == nnc.E_KV_FULL
    other = nnc.Pages.empty(3, 4, 16, 2, 128, torch.bfloat16, DEV)
    with pytest.raises(nnc.NncError) as e:
        m.decode_step_paged(other, tables, ln, tok)
    assert e.value.status == nnc.E_ARG
    with pytest.raises(nnc.NncError):
        m.pages_store(pages, tables, 0, 0, 0, 22)                             # the slot has 21
    with pytest.raises(nnc.NncError):
        m.pages_store(pages, tables, 4, 0)
    m.pages_store(pages, tables, 0, 0, 5, 0)


def beam_pages(nnc, shape, groups, width, prompt, steps, dtype, tokens=16):
    """Tables of a search: the prompt's full pages shared, everything behind them each beam's own."""
    full, per = prompt // tokens, -(-(prompt + steps) // tokens)
    pages = nnc.Pages.empty(shape.n_layers, groups * (full + width * (per - full)), tokens, shape.n_kv_heads, 128, dtype, DEV)
    ids = np.random.default_rng(2).permutation(pages.n_pages).astype(np.int32).reshape(groups, -1)
    t = np.zeros((groups, width, per), np.int32)
    t[:, :, :full] = ids[:, None, :full]
    t[:, :, full:] = ids[:, full:].reshape(groups, width, per - full)
    return pages, torch.from_numpy(t.reshape(groups * width, per)).to(DEV)


def begin(nnc, shape, groups, width, prompt, steps, dtype, blob=None):
    blob = synth.make_blob(shape, weight_std=0.05) if blob is None else blob
    m = nnc.Model(shape, blob, groups, 96)
    pages, tables = beam_pages(nnc, shape, groups, width, prompt, steps, dtype)
    logits = []
    for g in range(groups):
        lg, _ = m.prefill(g, synth.tokens(prompt, shape.vocab, stream=g))
        logits.append(lg)
        m.pages_store(pages, tables, g * width, g)
    return blob, m, pages, tables, torch.stack(logits), torch.full((groups * width,), prompt, dtype=torch.int32, device=DEV)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float8_e4m3fn, torch.int8])
@pytest.mark.parametrize("groups,width,prompt", [(1, 4, 37), (3, 3, 32), (2, 5, 15)])
def test_a_search_is_its_operators_one_by_one(nnc, dtype, groups, width, prompt):
    """nnc_decode_beam in one call and in two, against steps, selections and reorderings called in turn: the same bits."""
    steps, shape, eos = 9, SMALL_BF16, 5
    blob, m, pages, tables, logits, lens = begin(nnc, shape, groups, width, prompt, steps, dtype)
    tables0 = tables.clone()
    toks, pars, scores, ended = m.decode_beam(pages, tables, lens, steps, first_logits=logits, width=width, eos=eos)
    assert lens.tolist() == [prompt + steps - 1] * (groups * width)

    _, m2, pages2, tables2, logits2, lens2 = begin(nnc, shape, groups, width, prompt, steps, dtype, blob)
    assert torch.equal(tables0, tables2) and torch.equal(logits, logits2)
    t1, p1, s1, e1 = m2.decode_beam(pages2, tables2, lens2, 4, first_logits=logits2, width=width, eos=eos)
    t2, p2, s2, e2 = m2.decode_beam(pages2, tables2, lens2, steps - 4, tokens=t1[-1].contiguous(), scores=s1, finished=e1, eos=eos)
    assert torch.equal(torch.cat([t1, t2]), toks) and torch.equal(torch.cat([p1, p2]), pars) and torch.equal(s2, scores) and torch.equal(e2, ended)
    assert torch.equal(tables2, tables)

    _, m3, pages3, tables3, logits3, lens3 = begin(nnc, shape, groups, width, prompt, steps, dtype, blob)
    sc = torch.full((groups, width), -math.inf, device=DEV)
    sc[:, 0] = 0
    fin = torch.zeros((groups, width), dtype=torch.bool, device=DEV)
    lg = logits3[:, None].expand(groups, width, shape.vocab).contiguous()
    for step in range(steps):
        tok, par, sc, fin = nnc.beam_select(lg, sc, fin, eos)
        pages3.reorder(tables3, tables3, lens3, par)
        assert torch.equal(tok, toks[step]) and torch.equal(par, pars[step])
        if step + 1 < steps:
            lg, _ = m3.decode_step_paged(pages3, tables3, lens3, tok.reshape(-1))
            lg = lg.unflatten(0, (groups, width))
    assert torch.equal(sc, scores) and torch.equal(fin, ended) and torch.equal(tables3, tables)


@pytest.mark.parametrize("shape", [SMALL_BF16, SMALL_F32], ids=lambda s: s.name)
def test_scores_of_a_search_are_the_oracles(nnc, shape):
    """Every hypothesis read back along its parents: the sum of its log-probabilities by the oracle, token by token, is its score,
    within the logits' bound (4e-3) twice per step; and its first beam is at least the greedy one."""
    width, prompt, steps = 4, 21, 7
    blob, m, pages, tables, logits, lens = begin(nnc, shape, 1, width, prompt, steps, POOL[shape.dtype])
    toks, pars, scores, _ = (x.cpu().numpy() for x in m.decode_beam(pages, tables, lens, steps, first_logits=logits, width=width))
    o = oracle.from_shape(shape, blob, 1, 96)
    flags = oracle_flags(shape)
    prompt_toks = synth.tokens(prompt, shape.vocab, stream=0)
    seen = set()
    for b in range(width):
        hyp, at = [], b
        for step in reversed(range(steps)):
            hyp.append(int(toks[step, 0, at]))
            at = int(pars[step, 0, at])
        hyp.reverse()
        seen.add(tuple(hyp))
        o.kv_reset(0)
        lo, _ = o.prefill(0, prompt_toks, flags)
        total = 0.0
        for t in hyp:
            x = np.asarray(lo, np.float64).reshape(-1)
            total += x[t] - (x.max() + math.log(np.exp(x - x.max()).sum()))
            lo, _ = o.step_token(0, t, flags)
        assert abs(total - scores[0, b]) <= 2 * steps * 4e-3, (b, total, scores[0, b])
    assert len(seen) == width and (np.diff(scores[0]) <= 0).all()


def test_a_search_of_one_beam_is_greedy(nnc):
    shape, steps = SMALL_G4, 12
    blob, m, pages, tables, logits, lens = begin(nnc, shape, 2, 1, 30, steps, torch.bfloat16)
    toks, pars, _, _ = m.decode_beam(pages, tables, lens, steps, first_logits=logits, width=1)
    first = logits.argmax(-1).tolist()
    want, _ = m.decode_greedy([0, 1], first, steps - 1)
    assert toks[0, :, 0].tolist() == first and torch.equal(toks[1:, :, 0], want) and (pars == 0).all()


def test_steps_and_searches_in_a_callers_graph(nnc):
    """A step and a search step captured on the model's stream and replayed over a page boundary, eager work in between, against
    the same calls on a second model (one max_len for all of them: the same launches)."""
    shape, prompt, steps, width = SMALL_BF16, 28, 7, 3
    blob = synth.make_blob(shape, weight_std=0.05)
    sides = []
    for _ in range(2):
        _, m, pages, tables, logits, lens = begin(nnc, shape, 1, width, prompt, steps + 2, torch.bfloat16, blob)
        toks, _, scores, fin = m.decode_beam(pages, tables, lens, 1, first_logits=logits, width=width)
        sides.append(dict(m=m, pages=pages, tables=tables, lens=lens, tok=toks[-1].clone(), scores=scores, fin=fin))
    a, b = sides

    def call(s):
        return s["m"].decode_beam(s["pages"], s["tables"], s["lens"], 1, tokens=s["tok"], scores=s["scores"], finished=s["fin"], max_len=prompt + steps)

    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=a["m"].stream):
        got = call(a)
    for _ in range(steps - 1):
        graph.replay()
        want = call(b)
        torch.cuda.synchronize()
        for x, y in zip(got, want):
            assert torch.equal(x, y)
        assert torch.equal(a["tables"], b["tables"]) and torch.equal(a["lens"], b["lens"])
        for s, out in ((a, got), (b, want)):
            s["tok"].copy_(out[0][-1])
            s["scores"].copy_(out[2])
            s["fin"].copy_(out[3])
        a["m"].decode_step([0], [1])                      # (other work of the model between the replays)
        torch.cuda.synchronize()
    step = torch.cuda.CUDAGraph()
    with torch.cuda.graph(step, stream=a["m"].stream):
        logits, nxt = a["m"].decode_step_paged(a["pages"], a["tables"], a["lens"], a["tok"].reshape(-1), max_len=prompt + steps + 1)
    for _ in range(2):
        step.replay()
        wl, wn = b["m"].decode_step_paged(b["pages"], b["tables"], b["lens"], b["tok"].reshape(-1), max_len=prompt + steps + 1)
        torch.cuda.synchronize()
        assert torch.equal(logits, wl) and torch.equal(nxt, wn) and torch.equal(a["lens"], b["lens"])


def test_searches_that_cannot_be_run_are_refused(nnc):
    shape, prompt = SMALL_BF16, 20
    blob, m, pages, tables, logits, lens = begin(nnc, shape, 1, 3, prompt, 12, torch.int8)
    tables0, lens0 = tables.clone(), lens.clone()

    def refused(status, **change):
        args = dict(n_steps=3, first_logits=logits, width=3, eos=2, max_len=prompt)
        args.update(change)
        with pytest.raises(nnc.NncError) as e:
            m.decode_beam(pages, tables, lens, **args)
        assert e.value.status == status

    refused(nnc.E_ARG, n_steps=0)
    refused(nnc.E_ARG, eos=shape.vocab)
    refused(nnc.E_ARG, eos=-2)
    refused(nnc.E_ARG, width=2)
    refused(nnc.E_ARG, first_logits=logits.double())
    refused(nnc.E_ARG, first_logits=None)
    refused(nnc.E_KV_FULL, n_steps=14)                    # two pages of 16 hold 32: prompt + 13 passes exceed them
    refused(nnc.E_KV_FULL, max_len=31)
    wide = torch.zeros((22, 2), dtype=torch.int32, device=DEV)
    with pytest.raises(nnc.NncError) as e:                # more beams than a step has columns
        m.decode_beam(pages, wide, torch.full((22,), 5, dtype=torch.int32, device=DEV), 2, first_logits=logits.expand(2, -1).contiguous(), width=11)
    assert e.value.status == nnc.E_ARG
    with pytest.raises(nnc.NncError) as e:
        m.decode_step_paged(pages, wide, torch.full((22,), 5, dtype=torch.int32, device=DEV), torch.zeros(22, dtype=torch.int32, device=DEV))
    assert e.value.status == nnc.E_ARG
    layer = nnc.Model(synth.ModelShape("layer", hidden=256, n_layers=2, n_q_heads=4, n_kv_heads=2, head_dim=128, ffn=512, vocab=0,
                                       has_embed_and_head=False, tied_lm_head=False, dtype=synth.F32),
                      synth.make_blob(synth.ModelShape("layer", hidden=256, n_layers=2, n_q_heads=4, n_kv_heads=2, head_dim=128, ffn=512, vocab=0,
                                                       has_embed_and_head=False, tied_lm_head=False, dtype=synth.F32)), 1, 32)
    with pytest.raises(nnc.NncError) as e:
        layer.decode_step_paged(pages, tables, lens, torch.zeros(3, dtype=torch.int32, device=DEV))
    assert e.value.status == nnc.E_STATE
    torch.cuda.synchronize()
    assert torch.equal(tables, tables0) and torch.equal(lens, lens0)   # nothing was enqueued


def test_profile_names_the_paged_kernels(nnc):
    _, m, pages, tables, logits, lens = begin(nnc, SMALL_BF16, 1, 3, 20, 4, torch.bfloat16)
    m.profile_begin()
    m.pages_store(pages, tables, 0, 0)
    m.decode_beam(pages, tables, lens, 2, first_logits=logits, width=3)
    got = {r["name"]: r["launches"] for r in m.profile_end()}
    assert got["page_rows"] == 2 and got["page_attention"] == 2 and got["beam"] == 5 and "attn_partial" not in got


def test_rows_of_a_failed_launch_are_not_stored(nnc):
    """A decode launch that gave up (a wait bounded to one poll, as in the tests of the slots) leaves rows that nobody may pass on."""
    shape = SMALL_BF16
    m = nnc.Model(shape, synth.make_blob(shape, weight_std=0.05), 16, 64)
    pages = nnc.Pages.empty(shape.n_layers, 4, 16, shape.n_kv_heads, 128, torch.bfloat16, DEV)
    tables = torch.arange(4, dtype=torch.int32, device=DEV).reshape(1, 4)
    for s in range(16):
        m.prefill(s, synth.tokens(9, shape.vocab, stream=s))
    m.pages_store(pages, tables, 0, 3)
    m.set_option(nnc.OPT_FUSE_NORM, 1)
    m.set_option(nnc.OPT_SPIN_LIMIT, 1)
    m.decode_greedy(list(range(16)), [1] * 16, 8)
    with pytest.raises(nnc.NncError) as e:
        m.synchronize()
    assert e.value.status == nnc.E_DEVICE
    with pytest.raises(nnc.NncError) as e:
        m.pages_store(pages, tables, 0, 3)
    assert e.value.status == nnc.E_DEVICE
