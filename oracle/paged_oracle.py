"""Plain forms, in 64 bits, of the paged key/value cache's operators.

A pool holds pages [n_pages, Hkv, page, hd]; codes is None for a pool of plain
elements, else the exponent bytes [n_pages, Hkv, page] of e4m3 codes. A batch is
row_start [B + 1], kv_len [B], pages [B, max_pages] (lists or arrays). Written
from the definitions, one sequence at a time.
"""
from __future__ import annotations

import math

import numpy as np


def e4m3_value(code: int) -> float:
    """The number an e4m3 code stands for: sign, 4 exponent bits (bias 7), 3 fraction bits; 0x7f is NaN."""
    sign = -1.0 if code & 0x80 else 1.0
    e, f = (code >> 3) & 15, code & 7
    if e == 15 and f == 7:
        return math.nan
    return sign * (math.ldexp(1 + f / 8, e - 7) if e else math.ldexp(f / 8, -6))


E4M3 = np.array([e4m3_value(c) for c in range(256)])


def e4m3_code(x: np.ndarray, limit: float = 448.0) -> np.ndarray:
    """Codes of the nearest e4m3 numbers, ties to the even code; |x| over `limit` (a code) saturates, NaN is 0x7f."""
    x = np.asarray(x, dtype=np.float64)
    mags = E4M3[:0x7f]  # ascending
    a = np.minimum(np.abs(x), limit)
    hi = np.minimum(np.searchsorted(mags, a), 0x7e)
    lo = np.maximum(hi - 1, 0)
    with np.errstate(invalid="ignore"):
        up, down = mags[hi] - a, a - mags[lo]
        code = np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
    code = code | np.where(np.signbit(x), 0x80, 0)
    return np.where(np.isnan(x), 0x7f, code).astype(np.uint8)


def row_exponent(row: np.ndarray) -> int:
    """Least e in [-126, ...] with the row's largest finite magnitude <= 448 * 2^e."""
    a = np.abs(np.asarray(row, dtype=np.float64))
    a = a[np.isfinite(a)]
    top = float(a.max()) if a.size else 0.0
    e = -126
    while top > math.ldexp(448.0, e):
        e += 1
    return e


def quantise(rows: np.ndarray):
    """rows [..., hd] -> (codes, exponent bytes [...]); with 2^120 codes up to 240, so that all of them widen to fp32."""
    rows = np.asarray(rows, dtype=np.float64)
    flat = rows.reshape(-1, rows.shape[-1])
    codes = np.empty(flat.shape, dtype=np.uint8)
    exps = np.empty(flat.shape[0], dtype=np.uint8)
    for i, r in enumerate(flat):
        e = row_exponent(r)
        codes[i] = e4m3_code(r * math.ldexp(1.0, -e), 240.0 if e == 120 else 448.0)
        exps[i] = e + 127
    return codes.reshape(rows.shape), exps.reshape(rows.shape[:-1])


def widen(codes: np.ndarray, exps: np.ndarray) -> np.ndarray:
    return E4M3[codes] * np.ldexp(1.0, exps.astype(np.int64) - 127)[..., None]


def rows_of(row_start, kv_len, b: int, max_rows: int):
    """(row, slot) of sequence b's rows that take part."""
    n = row_start[b + 1] - row_start[b]
    return [(row_start[b] + i, kv_len[b] - n + i) for i in range(min(n, max_rows))]


def sequence(pool, exps, pages_b, kv: int, page: int) -> np.ndarray:
    """The first kv slots of a sequence: [kv, Hkv, hd] in 64 bits."""
    out = np.zeros((kv, pool.shape[1], pool.shape[3]))
    for i in range(-(-kv // page)):
        p, m = pages_b[i], min(page, kv - i * page)
        x = pool[p, :, :m] if exps is None else widen(pool[p, :, :m], exps[p, :, :m])
        out[i * page:i * page + m] = np.swapaxes(x, 0, 1)
    return out


def attention(q, pool_k, pool_v, exps_k, exps_v, row_start, kv_len, pages, page: int, max_rows: int, window: int = 0):
    """out [n_rows, Hq, hd], NaN at rows that no sequence has, and the sums of weight times |value| there."""
    q = np.asarray(q, dtype=np.float64)
    n_rows, hq, hd = q.shape
    out, spread = np.full(q.shape, np.nan), np.zeros(q.shape)
    group = hq // pool_k.shape[1]
    for b in range(len(kv_len)):
        k = sequence(pool_k, exps_k, pages[b], kv_len[b], page)
        v = sequence(pool_v, exps_v, pages[b], kv_len[b], page)
        for r, p in rows_of(row_start, kv_len, b, max_rows):
            lo = max(0, p - window + 1) if window else 0
            if p < 0:
                out[r] = 0.0
                continue
            for h in range(hq):
                kk, vv = k[lo:p + 1, h // group], v[lo:p + 1, h // group]
                with np.errstate(all="ignore"):
                    s = kk @ q[r, h] / math.sqrt(hd)
                    w = np.exp(s - np.max(s))
                    w /= w.sum()
                    out[r, h] = w @ vv
                    spread[r, h] = w @ np.abs(vv)
    return out, spread
