"""Paged caches at the edges of their types and of a batch."""
import numpy as np
import pytest
import torch

import paper_2607_21291_amd as P
from oracle import paged_oracle as G

from gpu_util import announce
from paged_util import DT, Setup, attention_bound

pytestmark = pytest.mark.gpu

MARK = 9.0


def _run(dev, s, hq, window=0, q=None):
    q = s.rows(hq, seed=11) if q is None else q
    c, batch = s.device(dev)
    out = torch.full((s.n_rows, hq, s.hd), MARK, dtype=DT[s.dtype], device=dev)
    P.paged_attention(c, batch, q.to(dev), out, window=window)
    torch.cuda.synchronize()
    return q, out.cpu()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_codes_of_the_largest_numbers_read_back_finite(dev, dtype):
    """Rows whose largest number lies around 448 2^119 and 248 2^120, up to the type's largest, with and without an
    infinity: 240 2^120 is the most that comes back, and what attention over such values gives is finite."""
    top = torch.finfo(DT[dtype]).max
    edges = [1.5 * 2.0 ** 127, 1.75 * 2.0 ** 127, 1.765625 * 2.0 ** 127, 1.9375 * 2.0 ** 127, 3.38e38, top]
    rows = [torch.full((64,), float(e), dtype=torch.float64).to(DT[dtype]) for e in edges]
    for r in list(rows):
        x = r.clone()
        x[7], x[8], x[9] = float("inf"), float("-inf"), -1.0
        rows.append(x)
    x = torch.stack(rows)[:, None]
    n = x.shape[0]
    s = Setup([(n, n)], hkv=1, hd=64, page=16, dtype=dtype, cache="e4m3")
    announce(f"paged write of the largest numbers {dtype}")
    c, batch = s.device(dev)
    P.paged_cache_write(c, batch, x.to(dev), x.to(dev))
    k, v = (torch.empty_like(x, device=dev) for _ in range(2))
    P.paged_cache_read(c, batch, k, v)
    # one slot seen by each row, so that nothing but its value counts
    out = torch.empty(n, 1, 64, dtype=DT[dtype], device=dev)
    P.paged_attention(c, batch, torch.zeros_like(out), out, window=1)
    torch.cuda.synchronize()
    want = torch.from_numpy(G.widen(*G.quantise(x.double().numpy())))
    assert want.abs().max() == 240 * 2.0 ** 120
    for got in (k, v):
        assert torch.equal(got.cpu().double(), want)
    finite = torch.isfinite(x)
    # half a step: 2^-4 relative for normal codes, and the least codes (the -1) lie 2^-9 2^e apart, e at most 120
    off = (want - x.double()).abs()[finite] - (2.0 ** -4 * x.double().abs()[finite]).clamp_min(2.0 ** 110)
    assert off.max() <= 0
    assert torch.equal(out.cpu().double(), want)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows", [1, 10, 30, 100])  # times two heads: every form of the kernels
@pytest.mark.parametrize("hd", [32, 64, 128])
def test_values_that_are_not_finite_reach_every_row_that_sees_them(dev, dtype, rows, hd):
    """One infinite or NaN value, in slots of whole tiles and of the first and last: that dimension of every row is it
    (its weight is far from 0), the others are what they were."""
    kv, at = 700, (0, 130, 400, 700 - rows)
    for value in (float("inf"), float("-inf"), float("nan")):
        for i, slot in enumerate(at):
            s = Setup([(rows, kv), (1, 20)], hkv=1, hd=hd, page=16, dtype=dtype, cache=dtype)
            announce(f"paged attention {dtype} hd={hd} rows={rows}: {value} in slot {slot}")
            q = s.rows(2, seed=11)
            ref, spread = s.attention(q)
            s.v[s.pages[0, slot // 16], 0, slot % 16, 5 + i] = value
            got = _run(dev, s, 2, q=q)[1].double().numpy()
            seen, col = got[:rows, :, 5 + i], 5 + i
            assert np.all(np.isnan(seen) if np.isnan(value) else seen == value)
            got[:rows, :, col] = ref[:rows, :, col]
            assert np.all(np.abs(got - ref) <= attention_bound(s, q, ref, spread, 2 * rows <= 64))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows", [1, 10, 30, 100])
def test_scores_of_minus_infinity_weigh_nothing(dev, dtype, rows):
    """Keys of -inf under queries above 0 in all slots but some: rows attend to those; in all slots: zeros."""
    for kept in ([3, 350, 699 - rows], []):
        s = Setup([(rows, 700)], hkv=1, hd=64, page=16, dtype=dtype, cache=dtype)
        q = s.rows(2, seed=11).abs() + 0.125
        k = torch.stack([s.k[s.pages[0, j // 16], 0, j % 16] for j in kept]).double() if kept else None
        v = torch.stack([s.v[s.pages[0, j // 16], 0, j % 16] for j in kept]).double() if kept else None
        for j in set(range(700)) - set(kept):
            s.k[s.pages[0, j // 16], 0, j % 16] = float("-inf")
        announce(f"paged attention {dtype} rows={rows}: scores of -inf but in {kept}")
        got = _run(dev, s, 2, q=q)[1].double()
        if not kept:
            assert (got == 0).all()
            continue
        w = torch.softmax(q.double() @ k.t() / 8.0, -1)
        far = (got - w @ v).abs().numpy()
        # (the bound's score sum goes by the finite keys)
        assert np.all(far <= attention_bound(s, q, (w @ v).numpy(), (w @ v.abs()).numpy(), 2 * rows <= 64))


def _within_its_rows_bound(s, q, out, window=0):
    """Every sequence against the bound of its own rows times heads, whatever else is in the batch."""
    ref, spread = s.attention(q, window)
    got = out.double().numpy()
    group = q.shape[1] // s.hkv
    for b, (n, _) in enumerate(s.seqs):
        n = min(n, s.max_rows)
        rows = slice(s.row_start[b], s.row_start[b] + n)
        bound = attention_bound(s, q, ref[rows], spread[rows], n * group <= 64)
        far = np.abs(got[rows] - ref[rows]) - bound
        assert far.max(initial=-1.0) <= 0.0, f"sequence {b}, {n} rows of {group} heads: {far.max():.3e} over the bound"


@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
@pytest.mark.parametrize("window", [0, 200])
@pytest.mark.parametrize("hq,hkv,seqs", [
    (14, 2, [(3, 300), (200, 400), (1, 1500), (9, 90), (10, 200), (2, 2)]),
    (2, 2, [(40, 300), (64, 700), (65, 1300), (130, 130), (17, 2100), (16, 64)]),
    (20, 1, [(1, 300), (2, 1400), (3, 500), (100, 200), (4, 70)]),
    (40, 1, [(1, 300), (2, 200), (50, 90), (1, 2000)]),
    (70, 1, [(1, 300), (2, 200)]),
    (100, 100, [(50, 80), (100, 120), (64, 1100), (1, 9)]),
])
def test_precision_goes_by_the_sequences_own_rows(dev, cache, window, hq, hkv, seqs):
    """Up to 64 rows times heads have 16 bits of each weight beside chunks too."""
    s = Setup(seqs, hkv=hkv, hd=32 if hkv > 2 else 64, page=16, cache=cache, pad=1)
    announce(f"paged attention {cache} heads {hq}/{hkv} window {window}: precision by rows")
    q, out = _run(dev, s, hq, window=window)
    _within_its_rows_bound(s, q, out, window)
    assert (out[-1] == MARK).all()


@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
@pytest.mark.parametrize("hq,hkv", [(14, 2), (12, 12), (20, 1)])
def test_precision_does_not_go_by_the_batchs_bounds(dev, cache, hq, hkv):
    """A captured step of up to 512 rows that brings one token, or a few: 16 bits as well."""
    for n in (1, 3):
        s = Setup([(n, 1600)], hkv=hkv, hd=128, page=64, cache=cache, pad=512 - n, max_rows=512)
        announce(f"paged attention {cache} heads {hq}/{hkv}: {n} rows of up to 512")
        q, out = _run(dev, s, hq)
        _within_its_rows_bound(s, q, out)
        assert (out[n:] == MARK).all()
