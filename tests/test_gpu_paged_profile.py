"""What the profile of a model on pages counts."""
import pytest
import torch

from parity_util import SMALL_BF16
from test_gpu_paged_long import setup

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def nnc():
    from paper_2512_21571_amd import binding
    binding.lib()
    return binding


@pytest.mark.parametrize("dtype,row", [(torch.float32, 512), (torch.bfloat16, 256), (torch.int8, 132), (torch.float8_e4m3fn, 132)])
@pytest.mark.parametrize("max_len", [0, 2000])
def test_bytes_are_those_of_the_positions_that_are_there(nnc, dtype, row, max_len):
    """Two layers of two kv heads: K and V of every cached position and of the new one, with their scales, whatever bound the call
    names; a sequence that is not run (its token does not exist) reads nothing."""
    lens = [700, 20, 333]
    m, pages, tables, first = setup(nnc, SMALL_BF16, lens, dtype, 16, 4)
    ln = torch.tensor(lens, dtype=torch.int32, device=DEV)
    tok = torch.tensor([first[0], SMALL_BF16.vocab, first[2]], dtype=torch.int32, device=DEV)
    if max_len:
        tables = torch.cat([tables, torch.full((3, 128), -1, dtype=torch.int32, device=DEV)], 1).contiguous()
    m.profile_begin()
    m.pages_store(pages, tables, 1, 1)
    m.decode_step_paged(pages, tables, ln, tok, max_len=max_len)
    m.decode_step_paged(pages, tables, ln, tok, max_len=max_len)
    got = {r["name"]: r for r in m.profile_end()}
    positions = 701 + 334 + 702 + 335
    assert got["page_attention"]["launches"] == 4
    assert got["page_attention"]["bytes"] == 2 * positions * 2 * 2 * row
    assert got["page_attention"]["flops"] == 2 * positions * 4 * 4 * 128
    assert got["page_rows"]["bytes"] == 2 * 20 * 2 * 2 * (256 + row)
    assert ln.tolist() == [702, 20, 335]
