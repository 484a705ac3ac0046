"""Numbers that the paged calls of a model cannot pass on, refused before anything is allocated or called."""
import types

import pytest


@pytest.fixture(scope="module")
def nnc():
    from paper_2512_21571_amd import binding
    binding.lib()
    return binding


@pytest.fixture
def model(nnc, monkeypatch):
    """A model that has nothing to be called on: a call of the library fails the test."""
    import torch

    class Never:
        def __getattr__(self, name):
            raise AssertionError("called " + name)

    monkeypatch.setattr(nnc, "lib", lambda: Never())
    m = nnc.Model.__new__(nnc.Model)
    m.torch, m.V, m.h, m.stream = torch, 100, None, types.SimpleNamespace(device=torch.device("cpu"))
    m._empty = lambda shape, dtype: torch.empty(shape, dtype=dtype)
    m._before = m._after = lambda: None
    p = nnc.Pages.__new__(nnc.Pages)
    p.torch, p.device, p._i32, p.desc = torch, torch.device("cpu"), torch.int32, nnc.NncPages()
    tables, lens, tokens = torch.zeros((2, 4), dtype=torch.int32), torch.zeros(2, dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    return m, p, tables, lens, tokens


def refused(nnc, f, *args, **kw):
    with pytest.raises(nnc.NncError) as e:
        f(*args, **kw)
    assert e.value.status == nnc.E_ARG


@pytest.mark.parametrize("max_len", [-1, 1 << 31, 1 << 32, (1 << 32) + 5, -(1 << 32)])
def test_bounds_of_more_bits_than_their_field(nnc, model, max_len):
    """2^32 would arrive as 0, "no bound", and 2^32 + 5 as 5, which would turn every longer sequence into NaN."""
    import torch
    m, p, tables, lens, tokens = model
    refused(nnc, m.decode_step_paged, p, tables, lens, tokens, max_len=max_len)
    refused(nnc, m.decode_beam, p, tables, lens, 1, first_logits=torch.zeros((1, 100)), width=2, max_len=max_len)


@pytest.mark.parametrize("n_steps", [0, -1, 1 << 31, 1 << 32, (1 << 32) + 1])
def test_steps_of_a_search(nnc, model, n_steps):
    import torch
    m, p, tables, lens, tokens = model
    refused(nnc, m.decode_beam, p, tables, lens, n_steps, first_logits=torch.zeros((1, 100)), width=2)


def test_what_fits_goes_on(nnc, model):
    import torch
    m, p, tables, lens, tokens = model
    with pytest.raises(AssertionError, match="nnc_decode_step_paged"):
        m.decode_step_paged(p, tables, lens, tokens, max_len=7)
    with pytest.raises(AssertionError, match="nnc_decode_beam"):
        m.decode_beam(p, tables, lens, 3, first_logits=torch.zeros((1, 100)), width=2, max_len=(1 << 31) - 1)


def test_positions_between_two_positions(nnc, model, monkeypatch):
    """Position 2.7 is not position 2."""
    import torch
    _, p, tables, _, _ = model
    p.n_layers, p.n_kv_heads, p.head_dim, p._desc = 1, 2, 64, None
    x = torch.zeros((3, 2, 64))

    def called(*args):
        raise AssertionError("called")

    monkeypatch.setattr(nnc, "_enqueue", called)
    for seq, pos in ((0.5, 0), (0, 2.7), (0, float("nan")), (float("inf"), 0)):
        refused(nnc, p.append, 0, x, x, tables, seq, pos)
        refused(nnc, p.read, 0, tables, seq, pos, k=x)
    with pytest.raises(AssertionError, match="called"):
        p.append(0, x, x, tables, 1.0, 2)
