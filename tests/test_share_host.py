"""What the entry points of shared attention, verification of drafts, bounds and picks refuse, before anything reaches a GPU."""
import ctypes

import pytest

from test_pages_host import BAD_PAGES, BAD_TABLES, P, nnc, pages, query, ref, table  # noqa: F401


def share(nnc, **change):
    d = dict(width=2, prefix=P, max_own=48)
    d.update(change)
    return nnc.NncPageShare(**d)


def bounds(nnc, **change):
    d = dict(lo=P, hi=P)
    d.update(change)
    return nnc.NncPageBounds(**d)


def pick(nnc, **change):
    d = dict(q=P, dtype=nnc.BF16, n_q_heads=8, q_row_stride=1024, q_head_stride=128, lens=P, max_len=48, keep=2, first=1, last=1, tables_out=P, lens_out=P)
    d.update(change)
    return nnc.NncPick(**d)


def drafts(nnc, **change):
    d = dict(logits=P, draft_logits=P, dtype=nnc.F32, row_stride=100, draft_row_stride=100, n=2, k=3, vocab=100, drafts=P, counts=P, uniforms=P, temperatures=None,
             temperature=1.0, tokens_out=P, accepted_out=P)
    d.update(change)
    return nnc.NncDrafts(**d)


def refused_everywhere(nnc, f, calls, match=None):
    for call in calls:
        assert f(call) == nnc.E_ARG, call
    assert nnc.last_error()


def test_structures_match_the_header(nnc):
    assert [ctypes.sizeof(s) for s in (nnc.NncPageShare, nnc.NncPageBounds, nnc.NncPick, nnc.NncDrafts)] == [24, 16, 72, 112]


def test_bad_pools_and_tables(nnc):
    L, n = nnc.lib(), ctypes.c_size_t(7)
    k = pick(nnc)

    def call(p, t):
        got = [L.nnc_page_attention_shared(ref(p), 0, ref(t), ref(query(nnc)), ref(share(nnc)), P, 1 << 30, None),
               L.nnc_page_attention_shared_workspace(ref(p), ref(t), ref(query(nnc)), ref(share(nnc)), ctypes.byref(n)),
               L.nnc_page_attention_picked(ref(p), 0, ref(t), ref(query(nnc)), P, 1 << 30, None),
               L.nnc_page_attention_picked_workspace(ref(p), ref(t), ref(query(nnc)), ctypes.byref(n)),
               L.nnc_page_bound(ref(p), 0, ref(bounds(nnc)), ref(t), P, None, 0, 0, None),
               L.nnc_page_pick(ref(p), 0, ref(bounds(nnc)), ref(t), ref(k), P, 1 << 30, None),
               L.nnc_page_pick_workspace(ref(p), ref(t), ref(k), ctypes.byref(n))]
        return set(got)

    assert call(None, table(nnc)) == {nnc.E_ARG} == call(pages(nnc), None)
    for change in BAD_PAGES:
        assert call(pages(nnc, **change), table(nnc)) == {nnc.E_ARG}, change
    for change in BAD_TABLES:
        assert call(pages(nnc), table(nnc, **change)) == {nnc.E_ARG}, change
    assert n.value == 7


def test_bad_shared_rows(nnc):
    L, n = nnc.lib(), ctypes.c_size_t(7)

    def call(p=None, t=None, q=None, s=None, layer=0, ws=P, size=1 << 30):
        p, t, q, s = p or pages(nnc), t or table(nnc), q or query(nnc), s or share(nnc)
        return L.nnc_page_attention_shared(ref(p), layer, ref(t), ref(q), ref(s), ws, size, None)

    for change in (dict(dtype=3), dict(n_q_heads=0), dict(n_q_heads=7), dict(n_q_heads=1 << 20), dict(max_len=49), dict(scale=float("nan")), dict(scale=float("inf")),
                   dict(q=P + 1), dict(out=P + 1), dict(lens=P + 2), dict(window=5)):
        assert call(q=query(nnc, **change)) == nnc.E_ARG, change
        assert L.nnc_page_attention_shared_workspace(ref(pages(nnc)), ref(table(nnc)), ref(query(nnc, **change)), ref(share(nnc)), ctypes.byref(n)) == nnc.E_ARG, change
    for change in (dict(width=0), dict(width=65536), dict(width=3), dict(prefix=P + 2), dict(prefix=None, width=20000)):
        assert call(s=share(nnc, **change)) == nnc.E_ARG, change
        assert L.nnc_page_attention_shared_workspace(ref(pages(nnc)), ref(table(nnc)), ref(query(nnc)), ref(share(nnc, **change)), ctypes.byref(n)) == nnc.E_ARG, change
    assert call(q=query(nnc, n_q_heads=4096), s=share(nnc, width=40000), t=table(nnc, n_seqs=40000)) == nnc.E_ARG      # more rows of heads than a launch takes
    assert n.value == 7
    assert L.nnc_page_attention_shared(ref(pages(nnc)), 0, ref(table(nnc)), ref(query(nnc)), None, P, 1 << 30, None) == nnc.E_ARG
    assert L.nnc_page_attention_shared(ref(pages(nnc)), 0, ref(table(nnc)), None, ref(share(nnc)), P, 1 << 30, None) == nnc.E_ARG
    assert call(layer=2) == nnc.E_ARG
    for change in (dict(q=None), dict(out=None), dict(lens=None)):
        assert call(q=query(nnc, **change)) == nnc.E_ARG, change
    # parts of a long context are joined, which needs a workspace of the size that is asked for
    long_t, long_q = table(nnc, max_pages=1024), query(nnc, max_len=16000)
    assert L.nnc_page_attention_shared_workspace(ref(pages(nnc)), ref(long_t), ref(long_q), ref(share(nnc)), ctypes.byref(n)) == nnc.OK and n.value > 0
    for ws, size in ((None, 1 << 30), (P, n.value - 1), (P + 4, 1 << 30)):
        assert call(t=long_t, q=long_q, ws=ws, size=size) == nnc.E_ARG
    assert "workspace" in nnc.last_error()
    assert call(t=table(nnc, n_seqs=0), ws=None, size=0) == nnc.OK                                                     # nobody there
    assert L.nnc_page_attention_shared_workspace(ref(pages(nnc)), ref(table(nnc)), ref(query(nnc)), ref(share(nnc, max_own=0)), ctypes.byref(n)) == nnc.OK and n.value == 0


def test_bad_picked_attention(nnc):
    L, n = nnc.lib(), ctypes.c_size_t(7)
    p, t = pages(nnc), table(nnc)
    for q, tt in ((query(nnc, window=1), t), (query(nnc, dtype=4), t), (query(nnc), table(nnc, n_seqs=3)), (query(nnc, max_len=49), t), (query(nnc, n_q_heads=9), t)):
        assert L.nnc_page_attention_picked(ref(p), 0, ref(tt), ref(q), P, 1 << 30, None) == nnc.E_ARG
        assert L.nnc_page_attention_picked_workspace(ref(p), ref(tt), ref(q), ctypes.byref(n)) == nnc.E_ARG
    assert n.value == 7
    for change in (dict(q=None), dict(out=None), dict(lens=None)):
        assert L.nnc_page_attention_picked(ref(p), 0, ref(t), ref(query(nnc, **change)), P, 1 << 30, None) == nnc.E_ARG
    assert L.nnc_page_attention_picked(ref(p), 2, ref(t), ref(query(nnc)), P, 1 << 30, None) == nnc.E_ARG
    assert L.nnc_page_attention_picked(ref(p), 0, ref(table(nnc, max_pages=4096)), ref(query(nnc, max_len=0)), None, 0, None) == nnc.E_ARG
    assert L.nnc_page_attention_picked(ref(p), 0, ref(table(nnc, n_seqs=0)), ref(query(nnc)), None, 0, None) == nnc.OK


def test_bad_bounds(nnc):
    L, p, t = nnc.lib(), pages(nnc), table(nnc)

    def call(b=None, layer=0, lens=P, since=P, since0=0, max_new=0, t=t):
        return L.nnc_page_bound(ref(p), layer, ref(b or bounds(nnc)), ref(t), lens, since, since0, max_new, None)

    for change in (dict(lo=None), dict(hi=None), dict(lo=P + 8), dict(hi=P + 2)):
        assert call(bounds(nnc, **change)) == nnc.E_ARG, change
    assert L.nnc_page_bound(ref(p), 0, None, ref(t), P, None, 0, 0, None) == nnc.E_ARG
    for kw in (dict(layer=2), dict(lens=None), dict(lens=P + 2), dict(since=P + 1), dict(since=None, since0=-1), dict(max_new=49)):
        assert call(**kw) == nnc.E_ARG, kw
    assert call(t=table(nnc, n_seqs=0)) == nnc.OK


def test_bad_picks(nnc):
    L, p, t, n = nnc.lib(), pages(nnc), table(nnc), ctypes.c_size_t(7)
    for change in (dict(dtype=3), dict(n_q_heads=0), dict(n_q_heads=9), dict(max_len=49), dict(keep=0), dict(keep=65537), dict(last=0), dict(first=2), dict(first=0, last=3),
                   dict(first=0xffffffff, last=2), dict(q=P + 1), dict(lens=P + 2), dict(tables_out=P + 2), dict(lens_out=P + 1)):
        assert L.nnc_page_pick(ref(p), 0, ref(bounds(nnc)), ref(t), ref(pick(nnc, **change)), P, 1 << 30, None) == nnc.E_ARG, change
        assert L.nnc_page_pick_workspace(ref(p), ref(t), ref(pick(nnc, **change)), ctypes.byref(n)) == nnc.E_ARG, change
    assert n.value == 7
    for change in (dict(q=None), dict(lens=None), dict(tables_out=None), dict(lens_out=None)):
        assert L.nnc_page_pick(ref(p), 0, ref(bounds(nnc)), ref(t), ref(pick(nnc, **change)), P, 1 << 30, None) == nnc.E_ARG, change
    assert L.nnc_page_pick(ref(p), 0, ref(bounds(nnc, lo=None)), ref(t), ref(pick(nnc)), P, 1 << 30, None) == nnc.E_ARG
    assert L.nnc_page_pick(ref(p), 2, ref(bounds(nnc)), ref(t), ref(pick(nnc)), P, 1 << 30, None) == nnc.E_ARG
    assert L.nnc_page_pick_workspace(ref(p), ref(t), ref(pick(nnc)), ctypes.byref(n)) == nnc.OK and n.value > 0
    for ws, size in ((None, 1 << 30), (P, n.value - 1), (P + 8, 1 << 30)):
        assert L.nnc_page_pick(ref(p), 0, ref(bounds(nnc)), ref(t), ref(pick(nnc)), ws, size, None) == nnc.E_ARG
    assert L.nnc_page_pick(ref(p), 0, ref(bounds(nnc)), ref(table(nnc, n_seqs=0)), ref(pick(nnc)), None, 0, None) == nnc.OK


def test_bad_drafts(nnc):
    L, n = nnc.lib(), ctypes.c_size_t(7)
    assert L.nnc_draft_verify(None, P, 1 << 30, None) == nnc.E_ARG
    assert L.nnc_draft_verify_workspace(None, ctypes.byref(n)) == nnc.E_ARG and L.nnc_draft_verify_workspace(ref(drafts(nnc)), None) == nnc.E_ARG
    for change in (dict(dtype=3), dict(vocab=0), dict(vocab=1 << 31), dict(k=0xffffffff), dict(k=65536), dict(n=65536), dict(n=10000, k=3)):
        assert L.nnc_draft_verify_workspace(ref(drafts(nnc, **change)), ctypes.byref(n)) == nnc.E_ARG, change
        assert L.nnc_draft_verify(ref(drafts(nnc, **change)), P, 1 << 30, None) == nnc.E_ARG, change
    assert n.value == 7
    for change in (dict(logits=None), dict(drafts=None), dict(uniforms=None), dict(tokens_out=None), dict(accepted_out=None), dict(logits=P + 2), dict(draft_logits=P + 1),
                   dict(drafts=P + 2), dict(counts=P + 1), dict(uniforms=P + 2), dict(temperatures=P + 2), dict(tokens_out=P + 2), dict(accepted_out=P + 1),
                   dict(temperature=-0.5), dict(temperature=float("nan")), dict(temperature=float("inf"))):
        assert L.nnc_draft_verify(ref(drafts(nnc, **change)), P, 1 << 30, None) == nnc.E_ARG, change
    assert L.nnc_draft_verify_workspace(ref(drafts(nnc)), ctypes.byref(n)) == nnc.OK
    for ws, size in ((None, 1 << 30), (P, n.value - 1), (P + 8, 1 << 30)):
        assert L.nnc_draft_verify(ref(drafts(nnc)), ws, size, None) == nnc.E_ARG
    assert L.nnc_draft_verify(ref(drafts(nnc, n=0)), None, 0, None) == nnc.OK


def test_models_refuse_before_they_look_at_pages(nnc):
    assert nnc.lib().nnc_decode_step_drafts(None, ref(pages(nnc)), ref(table(nnc)), P, 0, 2, P, None, None, None) == nnc.E_ARG


@pytest.fixture
def pool(nnc, monkeypatch):
    """A pool on the CPU; a call that would reach the library fails the test."""
    import torch

    def never(*args):
        raise AssertionError("called")

    monkeypatch.setattr(nnc, "_enqueue", never)
    p = nnc.Pages.__new__(nnc.Pages)
    p.torch, p.device, p._i32, p.dtype = torch, torch.device("cpu"), torch.int32, nnc.BF16
    p.k = torch.zeros((2, 8, 2, 16, 64), dtype=torch.bfloat16)
    p.n_layers, p.n_pages, p.n_kv_heads, p.page_tokens, p.head_dim = p.k.shape
    p.desc = pages(nnc, dtype=nnc.BF16, head_dim=64, k_scale=None, v_scale=None)
    p._desc = ctypes.byref(p.desc)
    return p


def test_the_binding_refuses_wrong_tensors_and_numbers(nnc, pool):
    import torch
    z = lambda *shape, dtype=torch.int32: torch.zeros(shape, dtype=dtype)
    f = torch.float32
    good = dict(layer=1, q=z(2, 3, 4, 64, dtype=f), tables=z(6, 4), lens=z(2, 3), prefix=z(2), max_len=64, max_own=5)
    with pytest.raises(AssertionError):
        pool.attention_shared(**good)
    with pytest.raises(AssertionError):
        pool.attention_shared(**{**good, "tables": z(2, 3, 4)})
    with pytest.raises(AssertionError):
        pool.attention_shared(**{**good, "tables": z(2, 4), "prefix": None, "max_own": None})
    for change in (dict(layer=2), dict(layer=-1), dict(layer=1 << 32), dict(q=z(6, 4, 64, dtype=f)), dict(q=z(2, 3, 4, 32, dtype=f)), dict(q=z(2, 3, 4, 64, dtype=torch.float64)),
                   dict(tables=z(2, 4)), dict(tables=z(6, 4, dtype=torch.int64)), dict(tables=z(6, 8)[:, ::2]), dict(lens=z(3, 2)), dict(lens=z(2, 3, dtype=torch.int64)),
                   dict(lens=z(2, 6)[:, ::2]), dict(prefix=z(3)), dict(prefix=z(2, dtype=f)), dict(prefix=None), dict(max_len=1 << 32), dict(max_len=-1), dict(max_own=-1),
                   dict(max_own=1 << 32), dict(out=z(2, 3, 4, 64)), dict(q=z(4, 3, 4, 64, dtype=f)[::2])):
        with pytest.raises(nnc.NncError) as e:
            pool.attention_shared(**{**good, **change})
        assert e.value.status == nnc.E_ARG, change
    b = (z(2, 8, 2, 64, dtype=torch.bfloat16),) * 2
    good = dict(layer=1, bounds=b, tables=z(3, 4), lens=z(3), since=z(3), max_new=5)
    with pytest.raises(AssertionError):
        pool.bound(**good)
    for change in (dict(layer=2), dict(bounds=(b[0], b[1].float())), dict(bounds=(b[0][:1], b[1])), dict(lens=z(2)), dict(lens=z(3, dtype=torch.int64)), dict(since=z(2)), dict(since=1 << 31),
                   dict(since=0.5), dict(max_new=-1), dict(max_new=1 << 32), dict(tables=z(3))):
        with pytest.raises(nnc.NncError):
            pool.bound(**{**good, **change})
    good = dict(layer=1, bounds=b, q=z(3, 4, 64, dtype=f), tables=z(3, 4), lens=z(3), keep=2)
    with pytest.raises(AssertionError):
        pool.pick(**good)
    for change in (dict(layer=2), dict(q=z(3, 5, 64, dtype=f)), dict(q=z(2, 4, 64, dtype=f)), dict(keep=0), dict(keep=1 << 32), dict(keep=70000), dict(first=-1), dict(first=2), dict(last=0),
                   dict(max_len=65), dict(max_len=1 << 32), dict(lens=z(4))):
        with pytest.raises(nnc.NncError):
            pool.pick(**{**good, **change})
    good = dict(layer=1, q=z(3, 4, 64, dtype=f), tables=z(3, 2, 2), lens=z(3, 2))
    with pytest.raises(AssertionError):
        pool.attention(**good)
    for change in (dict(tables=z(3, 3, 2)), dict(lens=z(3)), dict(lens=z(2, 3)), dict(window=4), dict(q=z(2, 4, 64, dtype=f)), dict(max_len=33), dict(tables=z(3, 2, 4)[:, :, ::2])):
        with pytest.raises(nnc.NncError):
            pool.attention(**{**good, **change})
    with pytest.raises(nnc.NncError):
        nnc.draft_verify(z(1, 3, 30, dtype=f), z(1, 2), z(1, 3, dtype=f))          # not device memory
