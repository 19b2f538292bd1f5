"""Writing into paged caches and reading back: bit for bit the plain form's, whatever the strides, pages and lengths."""
import math

import numpy as np
import pytest
import torch

import paper_2607_21291_amd as P
from oracle import paged_oracle as G

from gpu_util import announce
from paged_util import DT, Setup

pytestmark = pytest.mark.gpu

KINDS = [("bf16", "bf16"), ("f32", "f32"), ("bf16", "e4m3"), ("f32", "e4m3")]
SEQS = {
    "tokens": [(1, 1), (1, 17), (1, 64), (1, 300)],
    "ragged": [(5, 5), (0, 9), (1, 33), (70, 71), (0, 0), (129, 400)],
    "more_rows_than_slots": [(9, 4), (3, 3), (2, 0)],
    "many": [(i % 3, 1 + i % 40 + i % 3) for i in range(150)],
}


def _bits(t):
    t = t.cpu()
    return t.view({1: torch.uint8, 2: torch.int16, 4: torch.int32}[t.element_size()])


def _expect(s, new_k, new_v):
    """The pools after the write, as bits, from the plain form."""
    outs = []
    for pool, exps, new in ((s.k, s.ke, new_k), (s.v, s.ve, new_v)):
        pool = pool.clone()
        exps = exps.clone() if exps is not None else None
        if exps is not None:
            codes, bytes_ = (torch.from_numpy(a) for a in G.quantise(new.double().numpy()))
        for b in range(len(s.seqs)):
            for r, p in G.rows_of(s.row_start, s.kv_len, b, s.max_rows):
                if p < 0:
                    continue
                page, place = s.pages[b, p // s.page], p % s.page
                if exps is None:
                    pool[page, :, place] = new[r]
                else:
                    pool[page, :, place] = codes[r]
                    exps[page, :, place] = bytes_[r]
        outs += [pool, exps]
    return outs


@pytest.mark.parametrize("dtype,cache", KINDS)
@pytest.mark.parametrize("hd", [32, 64, 128])
@pytest.mark.parametrize("name", list(SEQS))
def test_write(dev, dtype, cache, hd, name):
    page = {32: 16, 64: 64, 128: 256}[hd]
    s = Setup(SEQS[name], hkv=3, hd=hd, page=page, dtype=dtype, cache=cache, pad=4)
    announce(f"paged write {dtype} {cache} hd={hd} {name}")
    c, batch = s.device(dev)
    # columns of wider rows, as a QKV projection leaves them
    qkv = s.rows(10, seed=3)
    new_k, new_v = qkv[:, 4:7], qkv[:, 7:10]
    on = qkv.to(dev)
    P.paged_cache_write(c, batch, on[:, 4:7], on[:, 7:10])
    torch.cuda.synchronize()
    for got, want in zip((c.k, c.k_exp, c.v, c.v_exp), _expect(s, new_k, new_v)):
        if want is not None:
            assert torch.equal(_bits(got), _bits(want))


@pytest.mark.parametrize("dtype,cache", KINDS)
@pytest.mark.parametrize("hd", [32, 64, 128])
@pytest.mark.parametrize("name", list(SEQS))
def test_read(dev, dtype, cache, hd, name):
    page = {32: 128, 64: 16, 128: 32}[hd]
    s = Setup(SEQS[name], hkv=2, hd=hd, page=page, dtype=dtype, cache=cache, pad=3)
    announce(f"paged read {dtype} {cache} hd={hd} {name}")
    c, batch = s.device(dev)
    outs = [torch.full((s.n_rows, 2, hd), 7.0, dtype=DT[dtype], device=dev) for _ in range(2)]
    P.paged_cache_read(c, batch, *outs)
    torch.cuda.synchronize()
    k, v, ke, ve = s.oracle_pools()
    for got, pool, exps in zip(outs, (k, v), (ke, ve)):
        want = torch.full((s.n_rows, 2, hd), 7.0, dtype=torch.float64)
        for b in range(len(s.seqs)):
            x = torch.from_numpy(G.sequence(pool, exps, s.pages[b], s.kv_len[b], s.page))
            for r, p in G.rows_of(s.row_start, s.kv_len, b, s.max_rows):
                want[r] = x[p] if p >= 0 else 0.0
        assert torch.equal(got.cpu().double().nan_to_num(nan=1e30), want.nan_to_num(nan=1e30))


@pytest.mark.parametrize("dtype,cache", KINDS)
def test_more_rows_than_a_pass_of_the_grid(dev, dtype, cache):
    """Every workgroup comes round again, with rows of several sequences, rows of none and rows without a slot."""
    s = Setup([(2500, 2600), (0, 5), (2500, 2000), (1699, 1699)], hkv=5, hd=128, page=128, dtype=dtype, cache=cache,
              pad=200)
    announce(f"paged copies {dtype} {cache} of many rows")
    c, batch = s.device(dev)
    new_k, new_v = s.rows(5, seed=4), s.rows(5, seed=5)
    outs = [torch.full(new_k.shape, 7.0, dtype=DT[dtype], device=dev) for _ in range(2)]
    P.paged_cache_write(c, batch, new_k.to(dev), new_v.to(dev))
    P.paged_cache_read(c, batch, *outs)
    torch.cuda.synchronize()
    want = _expect(s, new_k, new_v)
    for got, bits in zip((c.k, c.k_exp, c.v, c.v_exp), want):
        if bits is not None:
            assert torch.equal(_bits(got), _bits(bits))
    for got, pool, exps in ((outs[0], want[0], want[1]), (outs[1], want[2], want[3])):
        back = torch.full(new_k.shape, 7.0, dtype=torch.float64)
        for b in range(len(s.seqs)):
            parts = (pool.numpy(), exps.numpy()) if exps is not None else (pool.double().numpy(), None)
            x = torch.from_numpy(G.sequence(*parts, s.pages[b], s.kv_len[b], s.page))
            for r, p in G.rows_of(s.row_start, s.kv_len, b, s.max_rows):
                back[r] = x[p] if p >= 0 else 0.0
        assert torch.equal(got.cpu().double(), back)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_every_code_and_odd_values(dev, dtype):
    """Rows around every border of the format: zeros, the least numbers, infinities, NaN, ties, each code times a power
    of two; and back, exactly."""
    hd = 128
    rows = [torch.zeros(hd), torch.full((hd,), 2.0 ** -126), torch.full((hd,), 2.0 ** -133)]
    every = torch.from_numpy(G.E4M3[:0x7f]).float()
    for e in (-100, -9, 0, 3, 60, 110):
        rows.append(torch.cat([every, torch.tensor([-448.0])]) * 2.0 ** e)
    mid = (every[1:] + every[:-1]) / 2  # ties
    rows.append(torch.cat([mid, torch.tensor([448.0, -448.0])]))
    rows.append(-rows[-1])
    rows.append(torch.cat([mid * (1 + 2.0 ** -7), torch.tensor([448.0, 0.0])]))
    rows.append(torch.cat([torch.tensor([math.inf, -math.inf, math.nan, -0.0]), torch.linspace(-3, 3, hd - 4)]))
    rows.append(torch.full((hd,), math.nan))
    rows.append(torch.full((hd,), -math.inf))
    rows.append(torch.full((hd,), 3.38e38))
    g = torch.Generator().manual_seed(5)
    for e in range(-130, 120, 10):
        rows.append(torch.randn(hd, generator=g) * 2.0 ** e)
    x = torch.stack(rows)[:, None].to(DT[dtype])
    n = x.shape[0]
    s = Setup([(n, n)], hkv=1, hd=hd, page=16, dtype=dtype, cache="e4m3")
    announce(f"paged write, odd values {dtype}")
    c, batch = s.device(dev)
    P.paged_cache_write(c, batch, x.to(dev), x.flip(0).contiguous().to(dev))
    back = [torch.empty(n, 1, hd, dtype=DT[dtype], device=dev) for _ in range(2)]
    P.paged_cache_read(c, batch, *back)
    torch.cuda.synchronize()
    for got, want in zip((c.k, c.k_exp, c.v, c.v_exp), _expect(s, x, x.flip(0))):
        g8, w8 = _bits(got), _bits(want)
        if got.dim() == 4:  # NaN has two codes
            g8, w8 = (torch.where((t & 0x7f) == 0x7f, torch.full_like(t, 0x7f), t) for t in (g8, w8))
        assert torch.equal(g8, w8)
    codes, exps = G.quantise(x.double().numpy())
    want = torch.from_numpy(G.widen(codes, exps))
    # 2^e of the least rows is below the format's normal numbers; there both round once
    assert torch.equal(back[0].cpu().nan_to_num(nan=9.0), want.to(DT[dtype]).nan_to_num(nan=9.0))


@pytest.mark.parametrize("dtype,cache", [("bf16", "bf16"), ("bf16", "e4m3")])
def test_head_major_rows_and_max_rows(dev, dtype, cache):
    """Strides of a decode cache [Hkv, cap, hd], and rows past max_rows left out."""
    s = Setup([(40, 50)], hkv=3, hd=64, page=32, dtype=dtype, cache=cache, max_rows=33)
    announce(f"paged head-major {cache}")
    c, batch = s.device(dev)
    cap = s.rows(3).transpose(0, 1).contiguous()  # [Hkv, cap, hd]
    on = cap.to(dev)
    P.paged_cache_write(c, batch, on.transpose(0, 1), on.transpose(0, 1))
    back = torch.full((3, 40, 64), -5.0, dtype=DT[dtype], device=dev)
    other = torch.full((40, 3, 64), -5.0, dtype=DT[dtype], device=dev)
    P.paged_cache_read(c, batch, back.transpose(0, 1), other)
    torch.cuda.synchronize()
    x = cap.transpose(0, 1)
    for got, want in zip((c.k, c.k_exp, c.v, c.v_exp), _expect(s, x, x)):
        if want is not None:
            assert torch.equal(_bits(got), _bits(want))
    want = x.double()
    if cache == "e4m3":
        want = torch.from_numpy(G.widen(*G.quantise(x.double().numpy())))
    want = want.to(DT[dtype])
    want[33:] = -5.0
    assert torch.equal(back.transpose(0, 1).cpu(), want) and torch.equal(other.cpu(), want)


def test_bad_tables_stay_inside_the_pool(dev):
    """Page numbers, lengths and row starts outside their ranges are clamped: what is around the pool and the rows
    stays as it was."""
    hkv, hd, page, n_pages, N = 2, 64, 16, 5, 20
    hull = [torch.full((n_pages + 2, hkv, page, hd), 3.0, dtype=torch.bfloat16, device=dev) for _ in range(2)]
    c = P.PagedCache(hull[0][1:-1], hull[1][1:-1])
    i32 = lambda a: torch.tensor(a, dtype=torch.int32, device=dev)
    batch = P.PagedBatch(i32([-7, 9, 4, 500]), i32([1 << 30, -5, 77]), i32([[-1, 99, 1 << 30], [0, 1, 2], [-9, 5, 6]]), N,
                         N)
    hull_rows = torch.full((N + 2, hkv, hd), 4.0, dtype=torch.bfloat16, device=dev)
    rows = hull_rows[1:-1]
    announce("paged copies with bad tables")
    P.paged_cache_write(c, batch, rows, rows)
    P.paged_cache_read(c, batch, rows, torch.empty_like(rows))
    q = torch.ones(N, 4, hd, dtype=torch.bfloat16, device=dev)
    hull_out = torch.full((N + 2, 4, hd), 5.0, dtype=torch.bfloat16, device=dev)
    P.paged_attention(c, batch, q, hull_out[1:-1])
    torch.cuda.synchronize()
    for h in hull:
        assert (h[0] == 3).all() and (h[-1] == 3).all()
    assert (hull_rows[0] == 4).all() and (hull_rows[-1] == 4).all()
    assert (hull_out[0] == 5).all() and (hull_out[-1] == 5).all()


def test_offsets_past_32_bits(dev):
    """A pool of over 2^32 bytes and 2^31 elements, used at its end."""
    hkv, hd, page = 8, 128, 256
    n_pages = (1 << 31) // (hkv * hd * page) + 40  # elements per pool: 2^31 and some
    c = P.PagedCache.empty(n_pages, hkv, page, hd, torch.bfloat16, dev)
    lens = [300, 513]
    pages = torch.tensor([[n_pages - 1, n_pages - 3, 0], [n_pages - 5, n_pages - 2, n_pages - 9]], dtype=torch.int32)
    i32 = lambda a: torch.tensor(a, dtype=torch.int32, device=dev)
    batch = P.PagedBatch(i32([0, 300, 813]), i32(lens), pages.to(dev), 813, 513)
    g = torch.Generator().manual_seed(1)
    x = torch.randn(813, hkv, hd, generator=g).to(torch.bfloat16).to(dev)
    announce("paged pool past 2^32 bytes")
    P.paged_cache_write(c, batch, x, -x)
    k, v = torch.empty_like(x), torch.empty_like(x)
    P.paged_cache_read(c, batch, k, v)
    one = P.PagedBatch(i32([0, 1, 2]), i32(lens), pages.to(dev), 2, 1)
    q = torch.randn(2, hkv, hd, generator=g).to(torch.bfloat16).to(dev)
    out = torch.empty_like(q)
    P.paged_attention(c, one, q, out)
    torch.cuda.synchronize()
    assert torch.equal(k, x) and torch.equal(v, -x)
    assert torch.equal(c.k[n_pages - 2, 3, 255], x[300 + 511, 3])
    for b, (lo, hi) in enumerate(((0, 300), (300, 813))):
        for h in range(hkv):
            s = (x[lo:hi, h].double() @ q[b, h].double()) / math.sqrt(hd)
            want = torch.softmax(s, 0) @ -x[lo:hi, h].double()
            # probabilities as hi and lo, one rounding of the result
            assert torch.allclose(out[b, h].double(), want, rtol=2.0 ** -8, atol=1e-3)
