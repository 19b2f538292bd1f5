"""Paged caches with more sequences than a workgroup keeps in LDS, and with so many and so wide page tables that the
token kernel's units are longer than 64 slots."""
import numpy as np
import pytest
import torch

import paper_2607_21291_amd as P
from oracle import paged_oracle as G

from gpu_util import announce
from paged_util import DT, Setup, attention_bound

pytestmark = pytest.mark.gpu

MARK = 9.0


def _bits(t):
    t = t.cpu()
    return t.view({1: torch.uint8, 2: torch.int16, 4: torch.int32}[t.element_size()])


@pytest.mark.parametrize("dtype,cache", [("bf16", "bf16"), ("bf16", "e4m3"), ("f32", "f32")])
@pytest.mark.parametrize("count", [1024, 1025, 2100])
def test_copies_of_more_sequences_than_lds_holds(dev, dtype, cache, count):
    """Up to 1024 sequences' arrays are looked up in LDS, those of more in memory: the same bytes either way, with
    sequences without rows, rows past max_rows and rows before the first slot."""
    seqs = [((b * 5) % 4, (b * 11) % 23) for b in range(count)]
    s = Setup(seqs, hkv=2, hd=32, page=16, dtype=dtype, cache=cache, pad=5, max_rows=2)
    announce(f"paged copies {dtype} {cache} of {count} sequences")
    c, batch = s.device(dev)
    k, v = s.rows(2, seed=4), s.rows(2, seed=5)
    back = [torch.full(k.shape, 7.0, dtype=DT[dtype], device=dev) for _ in range(2)]
    P.paged_cache_write(c, batch, k.to(dev), v.to(dev))
    P.paged_cache_read(c, batch, *back)
    torch.cuda.synchronize()
    for got, got_exp, pool, exps, new, out in ((c.k, c.k_exp, s.k, s.ke, k, back[0]), (c.v, c.v_exp, s.v, s.ve, v, back[1])):
        pool, exps = pool.clone(), exps.clone() if exps is not None else None
        codes, bytes_ = (torch.from_numpy(a) for a in G.quantise(new.double().numpy()))
        want = torch.full(new.shape, 7.0, dtype=torch.float64)
        for b in range(count):
            for r, p in G.rows_of(s.row_start, s.kv_len, b, s.max_rows):
                if p < 0:
                    want[r] = 0.0
                    continue
                page, place = s.pages[b, p // s.page], p % s.page
                if exps is None:
                    pool[page, :, place] = new[r]
                    want[r] = new[r].double()
                else:
                    pool[page, :, place], exps[page, :, place] = codes[r], bytes_[r]
                    want[r] = torch.from_numpy(G.widen(codes[r].numpy(), bytes_[r].numpy()))
        assert torch.equal(_bits(got), _bits(pool))
        if exps is not None:
            assert torch.equal(got_exp.cpu(), exps)
        assert torch.equal(out.cpu().double(), want)


@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
@pytest.mark.parametrize("window", [0, 1300])
@pytest.mark.parametrize("chunk", [False, True])
def test_units_of_more_than_64_slots(dev, cache, window, chunk):
    """8192 sequences of up to 2^24 slots: units of 256 slots, so that their number stays below 2^30. Five sequences
    have rows; the long ones are shared between workgroups and joined."""
    B, page = 8192, 256
    held = {0: (1, 5000), 63: (1, 3), 64: (2, 1500), 4000: (1, 9111), 8191: (1, 300)}
    if chunk:
        held[4001] = (90, 1900)
    held = dict(sorted(held.items()))
    s = Setup(list(held.values()), hkv=2, hd=64, page=page, cache=cache, pad=2)
    announce(f"paged attention {cache} window {window} chunk {chunk}: {B} sequences of wide tables")
    c, small = s.device(dev)
    kv_len = torch.zeros(B, dtype=torch.int32)
    rows = torch.zeros(B, dtype=torch.int32)
    table = torch.zeros(B, (1 << 24) // page, dtype=torch.int32, device=dev)
    for i, (b, (n, kv)) in enumerate(held.items()):
        rows[b], kv_len[b] = n, kv
        table[b, :s.max_pages] = small.pages[i]
    row_start = torch.zeros(B + 1, dtype=torch.int32)
    row_start[1:] = torch.cumsum(rows, 0)
    batch = P.PagedBatch(row_start.to(dev), kv_len.to(dev), table, s.n_rows, s.max_rows)
    q = s.rows(6, seed=11)
    out = torch.full(q.shape, MARK, dtype=q.dtype, device=dev)
    P.paged_attention(c, batch, q.to(dev), out, window=window)
    torch.cuda.synchronize()
    ref, spread = s.attention(q, window)
    got = out.cpu().double().numpy()
    assert np.all(got[-2:] == MARK)
    for i, (n, _) in enumerate(s.seqs):
        r = slice(s.row_start[i], s.row_start[i] + n)
        far = np.abs(got[r] - ref[r]) - attention_bound(s, q, ref[r], spread[r], 3 * n <= 64)
        assert far.max() <= 0.0, f"sequence {i}: {far.max():.3e} over the bound"
