"""Paged caches without a GPU: refusals of the C entry points and of the binding, struct layouts, and pins of the
64-bit plain forms. Nothing here launches a kernel."""
import ctypes
import math
import os
import subprocess

import numpy as np
import pytest
import torch

import paper_2607_21291_amd as P
from oracle import paged_oracle as G
from paper_2607_21291_amd import _binding as B
from paged_util import Setup

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = 0x100000  # never dereferenced
OK_BUT_NO_GPU = 5


def _gpu():
    return torch.cuda.is_available()


def _cache(**kw):
    base = dict(k=FAKE, v=FAKE, k_exp=None, v_exp=None, type=P.BF16, n_pages=10, n_kv_heads=2, page_size=16, head_dim=64,
                reserved=0)
    base.update(kw)
    return B._PagedCacheStruct(*base.values())


def _batch(**kw):
    base = dict(row_start=FAKE, kv_len=FAKE, pages=FAKE, B=3, max_pages=100, n_rows=40, max_rows=20)
    base.update(kw)
    return B._PagedBatchStruct(*base.values())


def _addr(s):
    return ctypes.addressof(s) if s is not None else None


def _copy(fn, cache=None, batch=None, dtype=P.BF16, k=FAKE, k_row=128, k_head=64, v=FAKE, v_row=128, v_head=64):
    c, b = cache or _cache(), batch or _batch()
    return getattr(P.lib(), fn)(_addr(c), _addr(b), dtype, k, k_row, k_head, v, v_row, v_head, None)


def _attend(cache=None, batch=None, dtype=P.BF16, Hq=4, q=FAKE, q_row=256, q_head=64, window=0, out=FAKE, o_row=256,
            o_head=64, ws=FAKE, ws_bytes=1 << 40):
    c, b = cache or _cache(), batch or _batch()
    return P.lib().dsf_paged_attention(_addr(c), _addr(b), dtype, Hq, q, q_row, q_head, window, out, o_row, o_head, ws,
                                       ws_bytes, None)


BAD_CACHE = [(dict(type=P.F32), 2), (dict(type=7), 2), (dict(head_dim=96), 2), (dict(head_dim=256), 2),
             (dict(page_size=8), 2), (dict(page_size=48), 2), (dict(page_size=512), 2), (dict(n_pages=0), 1),
             (dict(n_kv_heads=0), 1), (dict(n_kv_heads=2048), 2), (dict(reserved=1), 1), (dict(k=None), 1),
             (dict(v=None), 1), (dict(k=FAKE + 8), 1), (dict(k_exp=FAKE), 1), (dict(type=P.E4M3), 1),
             (dict(type=P.E4M3, k_exp=FAKE), 1), (dict(type=P.E4M3, v_exp=FAKE), 1)]
BAD_BATCH = [(dict(row_start=None), 1), (dict(kv_len=None), 1), (dict(pages=None), 1), (dict(B=-1), 1),
             (dict(B=65537), 2), (dict(n_rows=-1), 1), (dict(max_rows=-1), 1), (dict(max_pages=0), 1),
             (dict(max_pages=(1 << 20) + 1), 2), (dict(pages=FAKE + 2), 1)]


@pytest.mark.parametrize("kw,code", BAD_CACHE)
def test_bad_caches_are_refused(kw, code):
    c = _cache(**kw)
    assert _copy("dsf_paged_cache_write", cache=c) == code and P.last_error()
    assert _copy("dsf_paged_cache_read", cache=c) == code
    assert _attend(cache=c) == code


@pytest.mark.parametrize("kw,code", BAD_BATCH)
def test_bad_batches_are_refused(kw, code):
    b = _batch(**kw)
    assert _copy("dsf_paged_cache_write", batch=b) == code and P.last_error()
    assert _copy("dsf_paged_cache_read", batch=b) == code
    assert _attend(batch=b) == code


def test_null_structs_are_refused():
    c, b = _cache(), _batch()
    for args in ((None, _addr(b)), (_addr(c), None)):
        assert P.lib().dsf_paged_cache_write(*args, P.BF16, FAKE, 128, 64, FAKE, 128, 64, None) == 1
        assert P.lib().dsf_paged_attention(*args, P.BF16, 4, FAKE, 256, 64, 0, FAKE, 256, 64, FAKE, 1 << 40, None) == 1
        assert P.lib().dsf_paged_attention_workspace_size(*args, P.BF16, 4) == 0


@pytest.mark.parametrize("fn", ["dsf_paged_cache_write", "dsf_paged_cache_read"])
def test_bad_rows_of_the_copies(fn):
    for kw in (dict(k=None), dict(v=None), dict(k=FAKE + 8), dict(v=FAKE + 2), dict(k_row=-128), dict(k_row=100),
               dict(v_head=60), dict(k_row=1 << 50)):
        assert _copy(fn, **kw) == 1, kw
    assert _copy(fn, dtype=7) == 2
    assert _copy(fn, dtype=P.F32) == 2  # a bf16 pool
    # rows in one place can be read, not written
    if fn == "dsf_paged_cache_read":
        for kw in (dict(k_row=0), dict(v_head=0), dict(k_head=32), dict(v_row=64)):
            assert _copy(fn, **kw) == 1, kw


def test_bad_attention_arguments():
    for kw, code in [(dict(dtype=7), 2), (dict(dtype=P.F32), 2), (dict(Hq=3), 1), (dict(Hq=0), 1), (dict(q=None), 1),
                     (dict(q=FAKE + 4), 1), (dict(out=None), 1), (dict(out=FAKE + 8), 1), (dict(q_row=250), 1),
                     (dict(q_head=-64), 1), (dict(o_row=0), 1), (dict(o_head=32), 1), (dict(o_row=128), 1),
                     (dict(window=-1), 1), (dict(ws=None), 1), (dict(ws=FAKE + 16), 1), (dict(ws_bytes=255), 3)]:
        assert _attend(**kw) == code, kw
    assert _attend(batch=_batch(n_rows=1 << 26)) == 1  # n_rows * Hq
    c, b = _cache(), _batch()
    need = P.lib().dsf_paged_attention_workspace_size(_addr(c), _addr(b), P.BF16, 4)
    assert need > 256 and need % 256 == 0
    assert _attend(ws_bytes=need - 1) == 3


def test_workspace_size_needs_no_pointers_and_refuses_bad_arguments():
    size = P.lib().dsf_paged_attention_workspace_size
    c = _cache(k=None, v=None)
    b = _batch(row_start=None, kv_len=None, pages=None)
    c2, b2, c3 = _cache(), _batch(), _cache(head_dim=48)
    assert 0 < size(_addr(c), _addr(b), P.BF16, 4) == size(_addr(c2), _addr(b2), P.BF16, 4)
    assert size(_addr(c3), _addr(b), P.BF16, 4) == 0
    assert size(_addr(c), _addr(b), P.BF16, 5) == 0
    assert size(_addr(c), _addr(b), 9, 4) == 0


def test_empty_batches_are_no_ops():
    for kw in (dict(B=0), dict(n_rows=0), dict(max_rows=0)):
        b = _batch(row_start=None, kv_len=None, pages=None, **kw)
        c = _cache(k=None, v=None)
        assert _copy("dsf_paged_cache_write", cache=c, batch=b, k=None, v=None) == 0
        assert _copy("dsf_paged_cache_read", cache=c, batch=b, k=None, v=None) == 0
        assert _attend(cache=c, batch=b, q=None, out=None, ws=None, ws_bytes=0) == 0


@pytest.mark.skipif(_gpu(), reason="placeholder pointers must never reach a real GPU")
def test_good_arguments_reach_the_device_check():
    for kw in (dict(), dict(cache=_cache(type=P.E4M3, k_exp=FAKE, v_exp=FAKE + 1)),
               dict(cache=_cache(type=P.F32), dtype=P.F32)):
        assert _copy("dsf_paged_cache_write", **kw) == OK_BUT_NO_GPU
        assert _copy("dsf_paged_cache_read", **kw) == OK_BUT_NO_GPU
        assert _attend(**kw) == OK_BUT_NO_GPU
    assert _copy("dsf_paged_cache_write", k_row=0, k_head=0) == OK_BUT_NO_GPU  # one key for all rows
    # head-major rows, as a decode cache has them
    assert _copy("dsf_paged_cache_read", k_row=64, k_head=64 * 40, v_row=64, v_head=64 * 40) == OK_BUT_NO_GPU


def test_struct_layouts_match_the_header(tmp_path):
    src = tmp_path / "layout.cpp"
    src.write_text('#include <cstdio>\n#include <cstddef>\n#include "adadsf.h"\nint main(){\n'
                   ' std::printf("%zu %zu %zu %zu %zu %zu\\n", sizeof(dsf_paged_cache), offsetof(dsf_paged_cache, type),'
                   " offsetof(dsf_paged_cache, head_dim), sizeof(dsf_paged_batch), offsetof(dsf_paged_batch, B),"
                   " offsetof(dsf_paged_batch, max_rows));\n}\n")
    exe = tmp_path / "layout"
    res = subprocess.run(["g++", "-std=c++17", "-D__HIP_PLATFORM_AMD__", "-I", os.path.join(ROOT, "include"),
                          "-I", "/opt/rocm/include", str(src), "-o", str(exe)], capture_output=True, text=True)
    if res.returncode != 0:
        pytest.skip("cannot compile against the HIP headers here: " + res.stderr[:200])
    got = [int(v) for v in subprocess.run([str(exe)], capture_output=True, text=True).stdout.split()]
    c, b = B._PagedCacheStruct, B._PagedBatchStruct
    assert got == [ctypes.sizeof(c), c.type.offset, c.head_dim.offset, ctypes.sizeof(b), b.B.offset, b.max_rows.offset]


# ------------------------------------------------------------ the binding

def _cpu_pool(dtype=torch.bfloat16):
    return P.PagedCache.empty(4, 2, 16, 64, dtype, "cpu")


def _cpu_batch(n_rows=5):
    i = lambda *a: torch.tensor(a, dtype=torch.int32)
    return P.PagedBatch(i(0, 2, 5), i(7, 9), torch.zeros(2, 3, dtype=torch.int32), n_rows, 3)


def test_binding_refuses_what_does_not_fit():
    bf, f8, u8 = torch.bfloat16, torch.float8_e4m3fn, torch.uint8
    z = torch.zeros
    with pytest.raises(ValueError):
        P.PagedCache(z(4, 2, 16, 64, dtype=bf), z(4, 2, 16, 32, dtype=bf))
    with pytest.raises(ValueError):
        P.PagedCache(z(4, 2, 16, 64, dtype=bf), z(4, 2, 16, 64))
    with pytest.raises(ValueError):
        P.PagedCache(z(4, 2, 16, 64, dtype=torch.float16), z(4, 2, 16, 64, dtype=torch.float16))
    with pytest.raises(ValueError):
        P.PagedCache(z(4, 2, 16, 64).to(f8), z(4, 2, 16, 64).to(f8))
    with pytest.raises(ValueError):
        P.PagedCache(z(4, 2, 16, 64).to(f8), z(4, 2, 16, 64).to(f8), z(4, 2, 16, dtype=u8), z(4, 2, 8, dtype=u8))
    with pytest.raises(ValueError):
        P.PagedCache(z(4, 2, 16, 64, dtype=bf), z(4, 2, 16, 64, dtype=bf), z(4, 2, 16, dtype=u8), z(4, 2, 16, dtype=u8))
    with pytest.raises(ValueError):
        P.PagedCache(z(4, 16, 2, 64, dtype=bf).transpose(1, 2), z(4, 16, 2, 64, dtype=bf).transpose(1, 2))
    i = lambda *a: torch.tensor(a, dtype=torch.int32)
    t = torch.zeros(2, 3, dtype=torch.int32)
    for args in ((i(0, 2), i(7, 9), t), (i(0, 2, 5), i(7, 9), t[:1]), (i(0, 2, 5).long(), i(7, 9), t),
                 (i(0, 2, 5), i(7, 9), t.flatten())):
        with pytest.raises(ValueError):
            P.PagedBatch(*args, 5, 3)
    c, b = _cpu_pool(), _cpu_batch()
    rows = z(5, 2, 64, dtype=bf)
    for k, v in ((z(4, 2, 64, dtype=bf), rows), (rows, z(5, 4, 64, dtype=bf)), (rows, z(5, 2, 32, dtype=bf)),
                 (rows.flatten(1), rows), (rows, rows.float()), (z(5, 64, 2, dtype=bf).transpose(1, 2), rows),
                 (rows.half(), rows.half())):
        for f in (P.paged_cache_write, P.paged_cache_read):
            with pytest.raises(ValueError):
                f(c, b, k, v)
    q = z(5, 4, 64, dtype=bf)
    for qq, out in ((q[:4], q[:4]), (q, q[:, :2]), (q, q.float()), (q.half(), q.half())):
        with pytest.raises(ValueError):
            P.paged_attention(c, b, qq, out)


def test_strides_whose_extent_passes_64_bits_are_refused():
    """2^40 elements times 2^24 rows is 0 in 64 bits."""
    many = _batch(n_rows=(1 << 24) + 1)
    for fn in ("dsf_paged_cache_write", "dsf_paged_cache_read"):
        assert _copy(fn, batch=many, k_row=1 << 40) == 1
        assert _copy(fn, batch=many, v_row=1 << 40) == 1
    assert _attend(batch=many, q_row=1 << 40) == 1
    assert _attend(batch=many, o_row=1 << 40) == 1


def test_binding_refuses_numbers_past_32_bits():
    """The C structures would take their lower halves."""
    b = _cpu_batch()
    for n_rows, max_rows in ((5, 1 << 32), (1 << 32, 3), (-1, 3), (5, -1)):
        with pytest.raises(ValueError, match="2\\^31"):
            P.PagedBatch(b.row_start, b.kv_len, b.pages, n_rows, max_rows)
    q = torch.zeros(5, 4, 64, dtype=torch.bfloat16)
    for window in (-1, 1 << 31, (1 << 32) + 5):
        with pytest.raises(ValueError, match="window"):
            P.paged_attention(_cpu_pool(), b, q, q.clone(), window=window)


def test_binding_refuses_tensors_off_the_gpu():
    c, b = _cpu_pool(), _cpu_batch()
    rows, q = torch.zeros(5, 2, 64, dtype=torch.bfloat16), torch.zeros(5, 4, 64, dtype=torch.bfloat16)
    for call in (lambda: P.paged_cache_write(c, b, rows, rows), lambda: P.paged_cache_read(c, b, rows, rows.clone()),
                 lambda: P.paged_attention(c, b, q, q.clone())):
        with pytest.raises(ValueError, match="not on a GPU"):
            call()


# ---------------------------------------------------------- the plain forms

def test_e4m3_codes_match_torch():
    x = torch.cat([torch.linspace(-460, 460, 20001), torch.randn(5000) * 2.0 ** -7, torch.tensor([0.0, -0.0])])
    x = x.clamp(-448, 448)
    got = G.e4m3_code(x.double().numpy())
    np.testing.assert_array_equal(got, x.to(torch.float8_e4m3fn).view(torch.uint8).numpy())
    every = torch.arange(256, dtype=torch.int32).to(torch.uint8)
    np.testing.assert_array_equal(G.E4M3, every.view(torch.float8_e4m3fn).double().numpy())
    np.testing.assert_array_equal(G.e4m3_code(np.array([np.nan, np.inf, -np.inf, 1e9])), [0x7f, 0x7e, 0xfe, 0x7e])


def test_row_exponents():
    for top, e in [(448.0, 0), (448.5, 1), (896.0, 1), (449.0, 1), (1.75, -8), (1.7500001, -7), (1.0, -8), (0.0, -126),
                   (2.0 ** -140, -126), (3.4e38, 120)]:
        assert G.row_exponent(np.array([0.0, -top, math.nan, math.inf])) == e, top


def test_plain_attention_is_the_softmax_over_the_sequence():
    s = Setup([(3, 20), (0, 0), (5, 3)], hkv=2, hd=32, page=16, dtype="f32", cache="f32")
    q = s.rows(4)
    out, _ = s.attention(q)
    k, v, _, _ = s.oracle_pools()
    ks = np.concatenate([k[s.pages[0, 0]], k[s.pages[0, 1]]], axis=1)[:, :20]
    vs = np.concatenate([v[s.pages[0, 0]], v[s.pages[0, 1]]], axis=1)[:, :20]
    for i in range(3):
        for h in range(4):
            x = torch.from_numpy(ks[h // 2, :18 + i] @ q[i, h].double().numpy() / math.sqrt(32))
            np.testing.assert_allclose(out[i, h], torch.softmax(x, 0).numpy() @ vs[h // 2, :18 + i], rtol=1e-12)
    assert np.all(out[3:5] == 0) and np.all(out[5:] != 0)  # two rows before the first slot
