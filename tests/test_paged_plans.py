"""How the paged attention's launches are sized, as far as the workspace shows it, and batches that are none. Nothing
here launches a kernel."""
import ctypes

import pytest
import torch

import paper_2607_21291_amd as P
from paper_2607_21291_amd import _binding as B


def _need(hq, hkv, n_seqs, n_rows, max_rows, max_pages=64, hd=128):
    c = B._PagedCacheStruct(None, None, None, None, P.BF16, 1000, hkv, 64, hd, 0)
    b = B._PagedBatchStruct(None, None, None, n_seqs, max_pages, n_rows, max_rows)
    return P.lib().dsf_paged_attention_workspace_size(ctypes.addressof(c), ctypes.addressof(b), P.BF16, hq)


@pytest.mark.parametrize("hq,hkv", [(28, 4), (14, 2), (16, 16), (12, 1)])
def test_tokens_beside_chunks_have_a_whole_chip_too(hq, hkv):
    """Tokens alone go to one workgroup of eight waves on each of 256 CUs; beside chunks workgroups have four waves, so
    there are two of them. A share has two places per workgroup, of 16 rows. (So many rows that chunks are not split
    and need none.)"""
    place = 16 * (128 * 4 + 8)
    alone = _need(hq, hkv, 40, 40, 1)
    beside = _need(hq, hkv, 40, 1 << 20, 1 << 15)
    assert alone == 2 * (256 // hkv) * hkv * place
    assert beside == 2 * (512 // hkv) * hkv * place


def test_batches_of_other_dimensions_are_refused():
    i = lambda *a: torch.tensor(a, dtype=torch.int32)
    table = torch.zeros(1, 3, dtype=torch.int32)
    for args in ((i(0, 1), torch.tensor(7, dtype=torch.int32), table), (i(0, 1), i(7).view(1, 1), table),
                 (i(0, 1).view(1, 2), i(7), table), (i(0, 1), i(7), table[0])):
        with pytest.raises(ValueError, match="row_start"):
            P.PagedBatch(*args, 1, 1)
