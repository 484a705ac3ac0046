"""What the entry points of the paged cache and of the beam selection refuse, before anything reaches a GPU."""
import ctypes

import numpy as np
import pytest


@pytest.fixture(scope="module")
def nnc():
    from paper_2512_21571_amd import binding
    binding.lib()
    return binding


MEM = np.zeros(4096, np.uint8)
P = (MEM.ctypes.data + 255) // 256 * 256      # (never reached: every call below is refused)


def pages(nnc, **change):
    d = dict(struct_bytes=ctypes.sizeof(nnc.NncPages), dtype=nnc.I8, n_layers=2, n_pages=8, page_tokens=16, n_kv_heads=2, head_dim=128, k=P, v=P, k_scale=P, v_scale=P)
    d.update(change)
    return nnc.NncPages(**d)


def table(nnc, **change):
    d = dict(entries=P, n_seqs=4, max_pages=3)
    d.update(change)
    return nnc.NncPageTable(**d)


def rows(nnc, **change):
    d = dict(k=P, v=P, dtype=nnc.BF16, k_row_stride=256, k_head_stride=128, v_row_stride=256, v_head_stride=128, n=4, seq=P, pos=P)
    d.update(change)
    return nnc.NncPageRows(**d)


def query(nnc, **change):
    d = dict(q=P, out=P, dtype=nnc.BF16, n_q_heads=8, q_row_stride=1024, q_head_stride=128, out_row_stride=1024, out_head_stride=128, lens=P, max_len=48, scale=0.1)
    d.update(change)
    return nnc.NncPageQuery(**d)


def beam(nnc, **change):
    d = dict(logits=P, dtype=nnc.F32, row_stride=100, n_groups=2, width=3, vocab=100, scores=P, finished=P, eos=7, tokens_out=P, parents_out=P, scores_out=P, finished_out=P)
    d.update(change)
    return nnc.NncBeam(**d)


def ref(x):
    return ctypes.byref(x) if x is not None else None


BAD_PAGES = [dict(struct_bytes=4), dict(dtype=3), dict(dtype=6), dict(n_layers=0), dict(n_layers=1025), dict(n_pages=0), dict(n_pages=1 << 31), dict(page_tokens=0),
             dict(page_tokens=4097), dict(n_kv_heads=0), dict(n_kv_heads=1025), dict(head_dim=96), dict(head_dim=0), dict(k=None), dict(v=None), dict(k=P + 8), dict(v=P + 2),
             dict(k_scale=None), dict(v_scale=None), dict(dtype=1), dict(k_scale=P + 2)]
BAD_TABLES = [dict(entries=None), dict(entries=P + 2), dict(max_pages=0), dict(max_pages=1 << 28), dict(n_seqs=65536)]


@pytest.mark.parametrize("what", ["append", "read", "attention", "reorder"])
def test_bad_pools_and_tables(nnc, what):
    L = nnc.lib()

    def call(p, t):
        if what in ("append", "read"):
            r = rows(nnc)
            return getattr(L, "nnc_page_" + what)(ref(p), 0, ref(t), ref(r), None)
        if what == "attention":
            n = ctypes.c_size_t()
            assert L.nnc_page_attention_workspace(ref(p), ref(t), ref(query(nnc)), ctypes.byref(n)) == nnc.E_ARG
            return L.nnc_page_attention(ref(p), 0, ref(t), ref(query(nnc)), P, 1 << 30, None)
        return L.nnc_page_reorder(ref(p), ref(t), P, P, P, 2, None)

    assert call(None, table(nnc)) == nnc.E_ARG
    assert call(pages(nnc), None) == nnc.E_ARG
    for change in BAD_PAGES:
        assert call(pages(nnc, **change), table(nnc)) == nnc.E_ARG, change
    for change in BAD_TABLES:
        assert call(pages(nnc), table(nnc, **change)) == nnc.E_ARG, change
    assert nnc.last_error()


@pytest.mark.parametrize("what", ["append", "read"])
def test_bad_rows(nnc, what):
    f = getattr(nnc.lib(), "nnc_page_" + what)
    p, t = pages(nnc), table(nnc)
    assert f(ref(p), 2, ref(t), ref(rows(nnc)), None) == nnc.E_ARG
    assert f(ref(p), 0, ref(t), None, None) == nnc.E_ARG
    for change in (dict(dtype=3), dict(dtype=nnc.I8), dict(k=P + 1), dict(v=P + 1), dict(dtype=nnc.F32, k=P + 2), dict(seq=P + 2), dict(pos=P + 1), dict(n=0xffffffff),
                   dict(pos=None, pos0=-1), dict(pos=None, pos0=0x7fffffff), dict(k=None, v=None)):
        assert f(ref(p), 0, ref(t), ref(rows(nnc, **change)), None) == nnc.E_ARG, change
    if what == "append":
        assert f(ref(p), 0, ref(t), ref(rows(nnc, k=None)), None) == nnc.E_ARG
        assert f(ref(p), 0, ref(t), ref(rows(nnc, v=None)), None) == nnc.E_ARG
    assert f(ref(p), 0, ref(t), ref(rows(nnc, n=0, k=None, v=None)), None) == nnc.OK      # no rows: nothing to do


def test_bad_queries(nnc):
    L = nnc.lib()
    p, t = pages(nnc), table(nnc)
    n = ctypes.c_size_t(77)
    for change in (dict(dtype=3), dict(n_q_heads=0), dict(n_q_heads=7), dict(n_q_heads=1 << 20), dict(max_len=49), dict(scale=float("nan")), dict(scale=float("inf")),
                   dict(q=P + 1), dict(out=P + 1), dict(lens=P + 2)):
        q = query(nnc, **change)
        assert L.nnc_page_attention_workspace(ref(p), ref(t), ref(q), ctypes.byref(n)) == nnc.E_ARG, change
        assert L.nnc_page_attention(ref(p), 0, ref(t), ref(q), P, 1 << 30, None) == nnc.E_ARG, change
    assert n.value == 77
    assert L.nnc_page_attention_workspace(ref(p), ref(t), None, ctypes.byref(n)) == nnc.E_ARG
    assert L.nnc_page_attention_workspace(ref(p), ref(t), ref(query(nnc)), None) == nnc.E_ARG
    assert L.nnc_page_attention(ref(p), 2, ref(t), ref(query(nnc)), P, 1 << 30, None) == nnc.E_ARG
    for change in (dict(q=None), dict(out=None), dict(lens=None)):
        assert L.nnc_page_attention(ref(p), 0, ref(t), ref(query(nnc, **change)), P, 1 << 30, None) == nnc.E_ARG, change
    # a long sequence needs a workspace of the size that is asked for
    long, q = table(nnc, max_pages=4096, n_seqs=1), query(nnc, max_len=0)
    assert L.nnc_page_attention_workspace(ref(p), ref(long), ref(q), ctypes.byref(n)) == nnc.OK and n.value > 0
    for ws, size in ((None, 1 << 30), (P, n.value - 1), (P + 4, 1 << 30)):
        assert L.nnc_page_attention(ref(p), 0, ref(long), ref(q), ws, size, None) == nnc.E_ARG
    assert "workspace" in nnc.last_error()
    assert L.nnc_page_attention(ref(p), 0, ref(table(nnc, n_seqs=0)), ref(q), None, 0, None) == nnc.OK    # nobody there


def test_bad_reorderings(nnc):
    L = nnc.lib()
    p, t = pages(nnc), table(nnc)
    for width in (0, 3, 33):
        assert L.nnc_page_reorder(ref(p), ref(t), P, P, P, width, None) == nnc.E_ARG
    for args in ((None, P, P), (P, None, P), (P, P, None), (P + 2, P, P), (P, P + 2, P), (P, P, P + 1)):
        assert L.nnc_page_reorder(ref(p), ref(t), *args, 2, None) == nnc.E_ARG
    assert L.nnc_page_reorder(ref(p), ref(table(nnc, n_seqs=0)), None, None, None, 2, None) == nnc.OK


def test_reorderings_that_one_launch_cannot_do(nnc):
    big, t = pages(nnc, n_layers=1024, n_kv_heads=1024, page_tokens=4096), table(nnc)
    assert nnc.lib().nnc_page_reorder(ref(big), ref(t), P, P, P, 2, None) == nnc.E_ARG
    assert "one call" in nnc.last_error()


def test_bad_selections(nnc):
    L = nnc.lib()
    n = ctypes.c_size_t()
    assert L.nnc_beam_select(None, P, 1 << 30, None) == nnc.E_ARG
    assert L.nnc_beam_select_workspace(None, ctypes.byref(n)) == nnc.E_ARG
    assert L.nnc_beam_select_workspace(ref(beam(nnc)), None) == nnc.E_ARG
    for change in (dict(width=0), dict(width=33), dict(vocab=0), dict(vocab=1 << 31), dict(dtype=3), dict(n_groups=30000)):
        assert L.nnc_beam_select_workspace(ref(beam(nnc, **change)), ctypes.byref(n)) == nnc.E_ARG, change
        assert L.nnc_beam_select(ref(beam(nnc, **change)), P, 1 << 30, None) == nnc.E_ARG, change
    for change in (dict(logits=None), dict(scores=None), dict(tokens_out=None), dict(parents_out=None), dict(scores_out=None), dict(eos=-2), dict(eos=100), dict(eos=-1),
                   dict(logits=P + 2), dict(scores=P + 1), dict(tokens_out=P + 1), dict(parents_out=P + 2), dict(scores_out=P + 2)):
        assert L.nnc_beam_select(ref(beam(nnc, **change)), P, 1 << 30, None) == nnc.E_ARG, change
    assert L.nnc_beam_select_workspace(ref(beam(nnc)), ctypes.byref(n)) == nnc.OK
    for ws, size in ((None, 1 << 30), (P, n.value - 1), (P + 8, 1 << 30)):
        assert L.nnc_beam_select(ref(beam(nnc)), ws, size, None) == nnc.E_ARG
    assert L.nnc_beam_select(ref(beam(nnc, n_groups=0)), None, 0, None) == nnc.OK


def test_models_refuse_before_they_look_at_pages(nnc):
    L = nnc.lib()
    p, t = pages(nnc), table(nnc)
    assert L.nnc_pages_store(None, ref(p), ref(t), 0, 0, 0, 1) == nnc.E_ARG
    assert L.nnc_decode_step_paged(None, ref(p), ref(t), P, 0, P, None, None) == nnc.E_ARG
    assert L.nnc_decode_beam(None, ref(p), ref(nnc.NncBeamRun())) == nnc.E_ARG


def test_the_binding_refuses_wrong_tensors(nnc):
    import torch
    cpu = torch.zeros((1, 4, 2, 16, 64), dtype=torch.bfloat16)
    with pytest.raises(nnc.NncError):
        nnc.Pages(cpu, cpu)
    with pytest.raises(nnc.NncError):
        nnc.Pages(cpu[0], cpu[0])
    with pytest.raises(nnc.NncError):
        nnc.Pages(cpu.double(), cpu.double())
    with pytest.raises(nnc.NncError):
        nnc.beam_select(torch.zeros((1, 2, 30)), torch.zeros((1, 2)))


def test_structures_match_the_header(nnc):
    """Sizes as a C compiler lays the header's structures out (x86-64)."""
    assert [ctypes.sizeof(s) for s in (nnc.NncPages, nnc.NncPageTable, nnc.NncPageRows, nnc.NncPageQuery, nnc.NncBeam, nnc.NncBeamRun)] == [64, 16, 88, 80, 96, 96]


def test_calls_run_on_the_device_of_their_tensors(nnc, monkeypatch):
    """On stand-ins for torch's device and stream: the tensors' device is current during the call and the stream is that device's;
    an error status becomes an exception after the device is back."""
    import types
    state = {"now": 0, "calls": []}

    class device:
        def __init__(self, i):
            self.i = i

        def __enter__(self):
            self.before, state["now"] = state["now"], self.i

        def __exit__(self, *exc):
            state["now"] = self.before

    fake = types.SimpleNamespace(cuda=types.SimpleNamespace(device=device),
                                 _C=types.SimpleNamespace(_cuda_getDevice=lambda: state["now"], _cuda_getCurrentRawStream=lambda i: 1000 + i))
    monkeypatch.setattr(nnc, "_torch", fake)

    def f(*args):
        state["calls"].append((state["now"], args))
        return nnc.OK if args[0] == "fine" else nnc.E_ARG

    for index in (0, 3):
        nnc._enqueue(types.SimpleNamespace(index=index), f, "fine", 7)
        with pytest.raises(nnc.NncError):
            nnc._enqueue(types.SimpleNamespace(index=index), f, "wrong")
    assert state["now"] == 0
    assert state["calls"] == [(i, args) for i in (0, 3) for args in (("fine", 7, 1000 + i), ("wrong", 1000 + i))]


def test_numbers_that_the_structures_cannot_hold(nnc, monkeypatch):
    """A number of more bits than its field is refused, not cut down to another position, sequence, layer or token.  (A pool on the
    CPU, and nothing is called.)"""
    import torch

    def never(*args):
        raise AssertionError("called")

    monkeypatch.setattr(nnc, "_enqueue", never)
    p = nnc.Pages.__new__(nnc.Pages)
    p.torch, p.device, p._i32 = torch, torch.device("cpu"), torch.int32
    p.n_layers, p.n_pages, p.n_kv_heads, p.page_tokens, p.head_dim = 2, 8, 2, 16, 64
    p.desc = pages(nnc, dtype=nnc.BF16, head_dim=64, k_scale=None, v_scale=None)
    p._desc = ctypes.byref(p.desc)
    tables, lens = torch.zeros((2, 4), dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    x, q = torch.zeros((3, 2, 64)), torch.zeros((2, 4, 64))
    for layer, seq, pos in ((-1, 0, 0), (2, 0, 0), (1 << 32, 0, 0), (0, 1 << 32, 0), (0, 0, 1 << 32), (0, 0, 1 << 31), (0, -(1 << 32), 0)):
        with pytest.raises(nnc.NncError) as e:
            p.append(layer, x, x, tables, seq, pos)
        assert e.value.status == nnc.E_ARG
        with pytest.raises(nnc.NncError):
            p.read(layer, tables, seq, pos, k=x)
    for change in (dict(layer=-1), dict(layer=1 << 32), dict(max_len=1 << 32), dict(max_len=-1), dict(window=1 << 32), dict(window=-5)):
        with pytest.raises(nnc.NncError) as e:
            p.attention(**{**dict(layer=0, q=q, tables=tables, lens=lens), **change})
        assert e.value.status == nnc.E_ARG
    with pytest.raises(AssertionError):
        p.append(1, x, x, tables, 1, 60)
    with pytest.raises(AssertionError):
        p.attention(1, q, tables, lens, max_len=64, window=3)
