"""How the paged attention's launches are sized, as far as the workspace shows it. Nothing here launches a kernel."""
import ctypes

import pytest

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
