"""Attention over paged caches against its plain form in 64 bits, at the lengths, pages, head layouts and masks where
it can go wrong. Slots that no sequence has hold NaN, exponent bytes there 255, other rows of `out` a mark."""
import numpy as np
import pytest
import torch

import paper_2607_21291_amd as P
from oracle import paged_oracle as G

from gpu_util import announce
from paged_util import DT, Setup, attention_bound

pytestmark = pytest.mark.gpu

KINDS = [("bf16", "bf16"), ("f32", "f32"), ("bf16", "e4m3"), ("f32", "e4m3")]
MARK = 9.0


def _few(s, hq):
    """Whether every sequence of the batch has at most 64 rows times heads."""
    return min(s.max_rows, s.n_rows) * (hq // s.hkv) <= 64


def _run(dev, s, hq, window=0, q_scale=1.0, workspace=None):
    q = s.rows(hq, seed=11, scale=q_scale)
    c, batch = s.device(dev)
    out = torch.full((s.n_rows, hq, s.hd), MARK, dtype=DT[s.dtype], device=dev)
    P.paged_attention(c, batch, q.to(dev), out, window=window, workspace=workspace)
    torch.cuda.synchronize()
    return q, out.cpu()


def _check(s, q, out, window=0):
    ref, spread = s.attention(q, window)
    mine = ~np.isnan(ref[:, 0, 0]) if ref.size else np.zeros(0, dtype=bool)
    taken = np.zeros(s.n_rows, dtype=bool)
    for b in range(len(s.seqs)):
        for r, _ in G.rows_of(s.row_start, s.kv_len, b, s.max_rows):
            taken[r] = True
    np.testing.assert_array_equal(mine, taken)
    got = out.double().numpy()
    assert np.all(got[~taken] == MARK)
    # a sequence of few rows may be in a batch with chunks: the wider bound holds for both
    bound = attention_bound(s, q, ref, spread, _few(s, q.shape[1]))
    far = np.abs(got - ref)[taken] - bound[taken]
    assert np.all(np.isfinite(got[taken]))
    assert far.max(initial=-1.0) <= 0.0, f"worst over the bound: {far.max():.3e}"


SEQS = {
    "one": [(1, 1)],
    "tokens": [(1, 1), (1, 16), (1, 17), (1, 63), (1, 64), (1, 65), (1, 333)],
    "few": [(2, 2), (4, 70), (3, 200), (0, 40), (1, 0), (2, 1)],
    "chunks": [(130, 130), (65, 400), (1, 90), (0, 0), (7, 300), (200, 201)],
    "empty_rows": [(90, 20), (3, 1), (1, 0), (70, 0)],
}


@pytest.mark.parametrize("dtype,cache", KINDS)
@pytest.mark.parametrize("hd", [32, 64, 128])
@pytest.mark.parametrize("name", list(SEQS))
def test_lengths(dev, dtype, cache, hd, name):
    page = {32: 64, 64: 16, 128: 128}[hd]
    s = Setup(SEQS[name], hkv=2, hd=hd, page=page, dtype=dtype, cache=cache, pad=3)
    announce(f"paged attention {dtype} {cache} hd={hd} {name}")
    q, out = _run(dev, s, 6)
    _check(s, q, out)


@pytest.mark.parametrize("dtype,cache", KINDS)
@pytest.mark.parametrize("hq,hkv", [(1, 1), (5, 5), (14, 2), (16, 1), (17, 1), (40, 1), (70, 1), (24, 12)])
def test_head_layouts(dev, dtype, cache, hq, hkv):
    s = Setup([(1, 50), (1, 129), (2, 30), (1, 1)], hkv=hkv, hd=64, page=32, dtype=dtype, cache=cache)
    announce(f"paged attention {dtype} {cache} heads {hq}/{hkv}")
    q, out = _run(dev, s, hq)
    _check(s, q, out)
    s = Setup([(33, 100), (1, 40)], hkv=hkv, hd=128, page=16, dtype=dtype, cache=cache)
    announce(f"paged attention {dtype} {cache} heads {hq}/{hkv}, chunk")
    q, out = _run(dev, s, hq)
    _check(s, q, out)


@pytest.mark.parametrize("dtype,cache", KINDS)
@pytest.mark.parametrize("page", [16, 32, 64, 128, 256])
def test_page_sizes(dev, dtype, cache, page):
    for seqs in ([(1, page), (1, page + 1), (1, 2 * page - 1)], [(70, page + 70), (80, 3 * page + 5)]):
        s = Setup(seqs, hkv=1, hd=64, page=page, dtype=dtype, cache=cache)
        announce(f"paged attention {dtype} {cache} pages of {page}")
        q, out = _run(dev, s, 2)
        _check(s, q, out)


@pytest.mark.parametrize("dtype,cache", KINDS)
@pytest.mark.parametrize("window", [1, 5, 64, 100, 1000])
def test_windows(dev, dtype, cache, window):
    for seqs in ([(1, 1), (1, 64), (1, 700), (3, 90)], [(100, 700), (300, 300), (2, 99), (70, 30)]):
        s = Setup(seqs, hkv=2, hd=64, page=16, dtype=dtype, cache=cache, pad=1)
        announce(f"paged attention {dtype} {cache} window {window}")
        q, out = _run(dev, s, 4, window=window)
        _check(s, q, out, window=window)


@pytest.mark.parametrize("dtype,cache", KINDS)
@pytest.mark.parametrize("hd", [32, 64, 128])
def test_long_sequences_are_split(dev, dtype, cache, hd):
    """Few rows over thousands of slots: the work of one sequence is split and joined, beside short ones."""
    for seqs, hq in (([(1, 5000), (1, 3), (1, 2111)], 3), ([(100, 4000), (1, 3500), (70, 90)], 3)):
        s = Setup(seqs, hkv=1, hd=hd, page=256, dtype=dtype, cache=cache, pad=2)
        announce(f"paged attention {dtype} {cache} hd={hd} split {seqs}")
        q, out = _run(dev, s, hq)
        _check(s, q, out)
        q, out = _run(dev, s, hq, window=1500)
        _check(s, q, out, window=1500)


@pytest.mark.parametrize("dtype,cache", KINDS)
@pytest.mark.parametrize("hd", [32, 64, 128])
def test_chunks_that_end_around_a_turn(dev, dtype, cache, hd):
    """Tiles of 1 to 7 turns of 64 slots, the last one whole, a slot short of it and a slot more."""
    seqs = [(70, 64 * k + d) for k in range(2, 8) for d in (-1, 0, 1)] + [(70, 70), (70, 64), (70, 63)]
    s = Setup(seqs, hkv=1, hd=hd, page=32, dtype=dtype, cache=cache)
    announce(f"paged attention {dtype} {cache} hd={hd} turns")
    q, out = _run(dev, s, 2)
    _check(s, q, out)


@pytest.mark.parametrize("dtype,cache", KINDS)
@pytest.mark.parametrize("window", [500, 1100, 2500])
def test_splits_of_a_window(dev, dtype, cache, window):
    """A tile's splits share what its own rows see: windows that begin at any slot, beside a chunk that is its own
    whole context and one whose rows are more than its slots."""
    s = Setup([(150, 5000), (90, 2777), (200, 200), (100, 40)], hkv=1, hd=64, page=64, dtype=dtype, cache=cache)
    announce(f"paged attention {dtype} {cache} splits of a window {window}")
    q, out = _run(dev, s, 3, window=window)
    _check(s, q, out, window=window)


@pytest.mark.parametrize("dtype,cache", [("bf16", "bf16"), ("f32", "f32"), ("bf16", "e4m3")])
@pytest.mark.parametrize("count", [63, 64, 65, 130])
def test_many_sequences(dev, dtype, cache, count):
    """More sequences than a wave has lanes, some without rows; with and without chunks among them."""
    seqs = [((b * 7) % 3, 1 + (b * 37) % 150) for b in range(count)]
    s = Setup(seqs, hkv=2, hd=32, page=16, dtype=dtype, cache=cache, pad=5)
    announce(f"paged attention {dtype} {cache} {count} sequences")
    q, out = _run(dev, s, 4)
    _check(s, q, out)
    seqs[count // 2] = (140, 1500)
    s = Setup(seqs, hkv=2, hd=32, page=16, dtype=dtype, cache=cache)
    q, out = _run(dev, s, 4)
    _check(s, q, out)


@pytest.mark.parametrize("dtype,cache", KINDS)
def test_peaked_scores(dev, dtype, cache):
    """Queries of ten times the size: the softmax is nearly one slot's, the maximum moves along the sequence."""
    for seqs in ([(1, 600), (2, 77)], [(80, 700)]):
        s = Setup(seqs, hkv=1, hd=64, page=64, dtype=dtype, cache=cache)
        announce(f"paged attention {dtype} {cache} peaked")
        q, out = _run(dev, s, 3, q_scale=10.0)
        _check(s, q, out)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows", [3, 100])
@pytest.mark.parametrize("hd", [32, 64, 128])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), float("-inf")])
def test_hidden_slots_have_no_effect(dev, dtype, rows, hd, value):
    """NaN and infinite keys and values in a slot reach the rows that see it and no other: not the rows before it, and
    not the ones whose window is past it."""
    kv = 300
    for at, window in ((kv - 2, 0), (kv - rows // 2, 0), (kv - rows - 10, 8 if rows == 3 else 60)):
        for what in ("v", "k"):
            s = Setup([(rows, kv), (1, 20)], hkv=1, hd=hd, page=16, dtype=dtype, cache=dtype)
            clean = s.attention(s.rows(2, seed=11), window)[0]
            pool = getattr(s, what)
            pool[s.pages[0, at // 16], 0, at % 16, 5 if what == "v" else slice(None)] = value
            announce(f"paged attention {dtype} hd={hd} rows={rows} {what}={value} at {at} window={window}")
            q, out = _run(dev, s, 2, window=window)
            slot = kv - rows + np.arange(rows)
            sees = (slot >= at) & ((slot - window < at) if window else True)
            hidden = np.concatenate([~sees, [True]])
            got = out.double().numpy()
            ref, spread = s.attention(q, window)
            assert np.all(np.isfinite(got[hidden]))
            bound = attention_bound(s, q, clean, np.nan_to_num(spread, nan=9.0, posinf=9.0), _few(s, 2))
            np.testing.assert_array_less(np.abs(got - clean)[hidden], bound[hidden] + 1e-30)
            seen = np.flatnonzero(~hidden)
            if what == "v" and len(seen):
                assert np.all(np.isnan(got[seen][..., 5]) if np.isnan(value) else got[seen][..., 5] == value)
                rest = np.delete(got[seen], 5, axis=-1)
                assert np.all(np.isfinite(rest))
            elif len(seen) and np.isnan(value):
                assert np.all(np.isnan(got[seen]))


def test_infinities_of_both_signs_are_nan(dev):
    s = Setup([(100, 260)], hkv=1, hd=64, page=16)
    for at, x in ((200, float("inf")), (203, float("-inf"))):
        s.v[s.pages[0, at // 16], 0, at % 16, 7] = x
    announce("paged attention, infinities of both signs")
    _, out = _run(dev, s, 2)
    got, slot = out[:, 0, 7].float(), 160 + torch.arange(100)
    assert torch.isfinite(got[slot < 200]).all()
    assert (got[(slot >= 200) & (slot < 203)] == float("inf")).all()
    assert torch.isnan(got[slot >= 203]).all()


@pytest.mark.parametrize("dtype,cache", [("bf16", "bf16"), ("f32", "f32"), ("bf16", "e4m3")])
def test_strided_rows(dev, dtype, cache):
    """q as the columns of QKV rows, out as a slice of wider rows; head-major rows too."""
    hq, hkv, hd = 6, 2, 64
    for seqs in ([(1, 70), (2, 9)], [(90, 140)]):
        s = Setup(seqs, hkv=hkv, hd=hd, page=32, dtype=dtype, cache=cache, pad=2)
        q = s.rows(hq, seed=11)
        c, batch = s.device(dev)
        qkv = torch.zeros(s.n_rows, hq + 2 * hkv + 1, hd, dtype=DT[dtype], device=dev)
        qkv[:, :hq] = q.to(dev)
        wide = torch.full((s.n_rows, hq + 3, hd), MARK, dtype=DT[dtype], device=dev)
        announce(f"paged attention {dtype} {cache} strided")
        P.paged_attention(c, batch, qkv[:, :hq], wide[:, 2:2 + hq])
        major = torch.full((hq, s.n_rows, hd), MARK, dtype=DT[dtype], device=dev)
        P.paged_attention(c, batch, qkv[:, :hq].transpose(0, 1).contiguous().transpose(0, 1), major.transpose(0, 1))
        torch.cuda.synchronize()
        assert (wide[:, :2] == MARK).all() and (wide[:, 2 + hq:] == MARK).all()
        assert torch.equal(wide[:, 2:2 + hq], major.transpose(0, 1))
        _check(s, q, wide[:, 2:2 + hq].cpu())


@pytest.mark.parametrize("dtype,cache", KINDS)
def test_rows_past_max_rows_are_left_out(dev, dtype, cache):
    for cut in (1, 3, 70):
        s = Setup([(5, 40), (90, 200), (1, 7)], hkv=1, hd=64, page=16, dtype=dtype, cache=cache, max_rows=cut)
        announce(f"paged attention {dtype} {cache} max_rows={cut}")
        q, out = _run(dev, s, 2)
        _check(s, q, out)


def test_sequences_may_share_pages(dev):
    s = Setup([(1, 100), (1, 100), (80, 100)], hkv=2, hd=64, page=16, share=(0, 1))
    s.pages[2] = s.pages[0]
    announce("paged attention, shared pages")
    q, out = _run(dev, s, 4)
    _check(s, q, out)


@pytest.mark.parametrize("dtype,cache", KINDS)
def test_same_bits_again_and_on_another_stream(dev, dtype, cache):
    for seqs in ([(1, 3000), (1, 40), (2, 700)], [(90, 2000), (1, 900)]):
        s = Setup(seqs, hkv=2, hd=128, page=64, dtype=dtype, cache=cache)
        announce(f"paged attention {dtype} {cache} repeated")
        q, first = _run(dev, s, 6)
        ws = torch.full((P.paged_attention_workspace_size(*s.device(dev), P.F32 if dtype == "f32" else P.BF16, 6),), 255,
                        dtype=torch.uint8, device=dev)  # NaN, and never cleared
        _, again = _run(dev, s, 6, workspace=ws)
        assert torch.equal(first, again)
        c, batch = s.device(dev)
        on = q.to(dev)
        out = torch.full(first.shape, MARK, dtype=first.dtype, device=dev)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        P.paged_attention(c, batch, on, out, stream=side)
        side.synchronize()
        assert torch.equal(first, out.cpu())


@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
def test_captured_step_replays_with_other_lengths(dev, cache):
    """Write and attention captured once; between replays the rows, lengths and pages change, and eager work runs.
    Two graphs with a workspace each, replayed in turn."""
    hq, hkv, hd, page, B, cap = 6, 2, 64, 16, 3, 2048
    g = torch.Generator().manual_seed(3)
    pool_dtype = torch.float8_e4m3fn if cache == "e4m3" else torch.bfloat16
    n_pages = B * cap // page
    table = torch.randperm(n_pages, generator=g).to(torch.int32).view(B, -1).to(dev)

    def make():
        c = P.PagedCache.empty(n_pages, hkv, page, hd, pool_dtype, dev)
        c.k.view(torch.uint8).zero_(), c.v.view(torch.uint8).zero_()
        row_start = torch.zeros(B + 1, dtype=torch.int32, device=dev)
        batch = P.PagedBatch(row_start, torch.zeros(B, dtype=torch.int32, device=dev), table, 40, 33)
        ws = torch.empty(P.paged_attention_workspace_size(c, batch, P.BF16, hq), dtype=torch.uint8, device=dev)
        qkv = torch.zeros(40, hq + 2 * hkv, hd, dtype=torch.bfloat16, device=dev)
        return c, batch, ws, qkv, torch.zeros(40, hq, hd, dtype=torch.bfloat16, device=dev)

    def step(c, batch, ws, qkv, out):
        P.paged_cache_write(c, batch, qkv[:, hq:hq + hkv], qkv[:, hq + hkv:])
        P.paged_attention(c, batch, qkv[:, :hq], out, workspace=ws)

    announce(f"paged step captured {cache}")
    eager, graphs = make(), []
    for _ in range(2):
        st = make()
        step(*st)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step(*st)
        graphs.append((graph, st))
    lens = [0] * B
    for t, rows in enumerate([[20, 3, 0], [1, 1, 1], [33, 1, 5], [1, 0, 1], [2, 30, 1], [1, 1, 1]]):
        lens = [n + r for n, r in zip(lens, rows)]
        qkv = torch.randn(40, hq + 2 * hkv, hd, generator=g).to(torch.bfloat16).to(dev)
        starts = torch.tensor([0] + list(np.cumsum(rows)), dtype=torch.int32, device=dev)
        for c, batch, ws, buf, out in [eager] + [st for _, st in graphs]:
            batch.row_start.copy_(starts)
            batch.kv_len.copy_(torch.tensor(lens, dtype=torch.int32, device=dev))
            buf.copy_(qkv)
            out.fill_(MARK)
        announce(f"paged step replay {t}")
        step(*eager)
        for graph, _ in graphs:
            graph.replay()
        torch.cuda.synchronize()
        for _, st in graphs:
            assert torch.equal(st[4], eager[4]) and torch.equal(st[0].k.view(torch.uint8), eager[0].k.view(torch.uint8))
        assert (eager[4][sum(rows):] == MARK).all()


@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
def test_prefill_in_chunks_then_tokens(dev, cache):
    """The operators together: a prompt in chunks, then tokens, two sequences in one batch, each step's keys and values
    written and attended to. With bf16 pages the rows equal attention over the whole sequence in one call within both
    roundings; with codes, attention over what reading the pages back gives."""
    hq, hkv, hd, page, T = 6, 2, 64, 32, 150
    g = torch.Generator().manual_seed(9)
    q, k, v = (torch.randn(2, T, h, hd, generator=g).to(torch.bfloat16).to(dev) for h in (hq, hkv, hkv))
    pool = torch.float8_e4m3fn if cache == "e4m3" else torch.bfloat16
    n_pages = 2 * -(-T // page)
    c = P.PagedCache.empty(n_pages, hkv, page, hd, pool, dev)
    table = torch.randperm(n_pages, generator=g).to(torch.int32).view(2, -1).to(dev)
    i32 = lambda a: torch.tensor(a, dtype=torch.int32, device=dev)
    outs = torch.zeros(2, T, hq, hd, dtype=torch.bfloat16, device=dev)
    done = [0, 0]
    announce(f"paged prefill in chunks {cache}")
    for rows in ([64, 1], [70, 90], [1, 40], [15, 19]):
        at = [slice(d, d + r) for d, r in zip(done, rows)]
        done = [d + r for d, r in zip(done, rows)]
        step = [torch.cat([x[0, at[0]], x[1, at[1]]]) for x in (q, k, v)]
        batch = P.PagedBatch(i32([0, rows[0], sum(rows)]), i32(done), table, sum(rows), max(rows))
        P.paged_cache_write(c, batch, step[1], step[2])
        out = torch.empty_like(step[0])
        P.paged_attention(c, batch, step[0], out)
        outs[0, at[0]], outs[1, at[1]] = out[:rows[0]], out[rows[0]:]
    assert done == [T, T]
    whole = P.PagedBatch(i32([0, T, 2 * T]), i32([T, T]), table, 2 * T, T)
    kk, vv = (torch.empty(2 * T, hkv, hd, dtype=torch.bfloat16, device=dev) for _ in range(2))
    P.paged_cache_read(c, whole, kk, vv)
    torch.cuda.synchronize()
    kk, vv = kk.view(2, T, hkv, hd), vv.view(2, T, hkv, hd)
    if cache == "bf16":
        assert torch.equal(kk, k) and torch.equal(vv, v)
    major = [x.transpose(1, 2).contiguous() for x in (q, kk, vv)]
    ref = torch.empty(2, T, hq * hd, dtype=torch.bfloat16, device=dev)
    P.attention_forward(*major, ref)
    torch.cuda.synchronize()
    ref = ref.view(2, T, hq, hd).double()
    # per call: weights rounded to bf16 in numerator and denominator, one rounding of the result; |v| under 5
    assert (outs.double() - ref).abs().max() <= 2 * (2 * 2.0 ** -8 * 5 + 2.0 ** -8 * 5)
    s = torch.einsum("bqhd,bkhd->bhqk", q.cpu().double(), kk.cpu().double().repeat_interleave(hq // hkv, 2)) / hd ** 0.5
    s = s.masked_fill(torch.ones(T, T, dtype=torch.bool).triu(1), -np.inf).softmax(-1)
    want = torch.einsum("bhqk,bkhd->bqhd", s, vv.cpu().double().repeat_interleave(hq // hkv, 2))
    spread = torch.einsum("bhqk,bkhd->bqhd", s, vv.cpu().double().abs().repeat_interleave(hq // hkv, 2))
    far = (outs.cpu().double() - want).abs() - (2.0 ** -7 * 1.02 * spread + 2.0 ** -8 * want.abs())
    assert far.max() <= 0


def test_decode_cache_moves_into_pages(dev):
    """The caches that a prefill fills ([B, Hkv, cap, hd], as many slots as each layer keeps) into pages, each sequence
    by its strides, and attention of one token over them as over the cache itself."""
    import synthetic as S
    from gpu_util import make_desc, workload, workspace
    w = workload("qwen_bf16_small").replace(n_layers=1)
    B, T, cap, k = 2, 300, 320, 181
    dl = P.DeviceLayer(S.layer_weights(w, 0), dev)
    ck = [torch.zeros(B, w.n_kv_heads, cap, w.head_dim, dtype=torch.bfloat16, device=dev) for _ in range(2)]
    clen = torch.zeros(1, B, dtype=torch.int32, device=dev)
    x = S.hidden_states(w, batch=B, seq=T).to(dev).contiguous()
    announce("decode cache into pages")
    P.stack_prefill(make_desc(w), [dl.weights], [k], x, ck[:1], ck[1:], clen, workspace(w, B, T, k, dev))
    c = P.PagedCache.empty(B * 12, w.n_kv_heads, 16, w.head_dim, torch.bfloat16, dev)
    table = torch.randperm(B * 12, generator=torch.Generator().manual_seed(0)).to(torch.int32).view(B, 12).to(dev)
    zero_k = torch.tensor([0, k], dtype=torch.int32, device=dev)
    for b in range(B):
        batch = P.PagedBatch(zero_k, clen[0, b:b + 1].contiguous(), table[b:b + 1].contiguous(), k, k)
        P.paged_cache_write(c, batch, ck[0][b, :, :k].transpose(0, 1), ck[1][b, :, :k].transpose(0, 1))
    q = torch.randn(B, w.n_heads, w.head_dim, generator=torch.Generator().manual_seed(1)).to(torch.bfloat16).to(dev)
    out = torch.empty_like(q)
    batch = P.PagedBatch(torch.arange(B + 1, dtype=torch.int32, device=dev), clen[0].contiguous(), table, B, 1)
    P.paged_attention(c, batch, q, out)
    torch.cuda.synchronize()
    g = w.n_heads // w.n_kv_heads
    for b in range(B):
        for h in range(w.n_heads):
            kk, vv = (t[b, h // g, :k].double() for t in ck)
            p = torch.softmax(kk @ q[b, h].double() / w.head_dim ** 0.5, 0)
            far = (out[b, h].double() - p @ vv).abs() - (2.0 ** -14 * (p @ vv.abs()) + 2.0 ** -8 * (p @ vv).abs())
            assert far.max() <= 1e-6
