"""Batches on paged caches for the tests: pools whose unused slots hold what must not matter."""
import math

import numpy as np
import torch

import paper_2607_21291_amd as P
from oracle import paged_oracle as G

DT = {"f32": torch.float32, "bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn}
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}  # half a step, relative


class Setup:
    """Sequences [(rows, slots)] over a pool of random pages; slots that no sequence has are NaN (codes: the NaN code
    and the exponent byte 255)."""

    def __init__(self, seqs, hkv, hd, page, dtype="bf16", cache="bf16", pad=0, seed=0, poison=True, max_rows=None,
                 spare=2, share=None):
        g = torch.Generator().manual_seed(seed)
        self.dtype, self.cache, self.page, self.hkv, self.hd, self.seqs = dtype, cache, page, hkv, hd, seqs
        self.row_start = [0]
        for n, _ in seqs:
            self.row_start.append(self.row_start[-1] + n)
        self.n_rows = self.row_start[-1] + pad
        self.kv_len = [kv for _, kv in seqs]
        self.max_rows = max_rows if max_rows is not None else max([n for n, _ in seqs] + [1])
        held = [-(-kv // page) for kv in self.kv_len]
        self.max_pages = max(held + [1])
        self.n_pages = sum(held) + spare
        order = torch.randperm(self.n_pages, generator=g).tolist()
        self.pages = np.zeros((len(seqs), self.max_pages), dtype=np.int64)
        at = 0
        for b, m in enumerate(held):
            self.pages[b, :m] = order[at:at + m]
            at += m
        if share is not None:  # sequence share[1] reads share[0]'s pages
            self.pages[share[1]] = self.pages[share[0]]
        shape = (self.n_pages, hkv, page, hd)
        used = np.zeros((self.n_pages, page), dtype=bool)
        for b, kv in enumerate(self.kv_len):
            for i in range(held[b]):
                used[self.pages[b, i], :min(page, kv - i * page)] = True
        self.used = torch.from_numpy(used)
        self.k, self.ke = self._pool(shape, g, poison)
        self.v, self.ve = self._pool(shape, g, poison)

    def _pool(self, shape, g, poison):
        unused = ~self.used[:, None, :].expand(shape[:3])
        if self.cache == "e4m3":
            x = torch.randint(0, 127, shape, generator=g, dtype=torch.int32) | \
                (torch.randint(0, 2, shape, generator=g, dtype=torch.int32) << 7)
            x = x.to(torch.uint8)
            e = torch.randint(119, 122, shape[:3], generator=g, dtype=torch.int32).to(torch.uint8)
            if poison:
                x[unused] = 0x7f
                e[unused] = 255
            return x, e
        x = torch.randn(shape, generator=g).to(DT[self.cache])
        if poison:
            x[unused] = math.nan
        return x, None

    def rows(self, heads, seed=1, scale=1.0):
        g = torch.Generator().manual_seed(seed)
        return (torch.randn(self.n_rows, heads, self.hd, generator=g) * scale).to(DT[self.dtype])

    def device(self, dev):
        codes = self.cache == "e4m3"
        to = lambda t: t.to(dev)
        k, v = to(self.k), to(self.v)
        if codes:
            k, v = k.view(torch.float8_e4m3fn), v.view(torch.float8_e4m3fn)
        cache = P.PagedCache(k, v, to(self.ke) if codes else None, to(self.ve) if codes else None)
        i32 = lambda a: torch.tensor(np.asarray(a), dtype=torch.int32, device=dev)
        batch = P.PagedBatch(i32(self.row_start), i32(self.kv_len), i32(self.pages), self.n_rows, self.max_rows)
        return cache, batch

    def oracle_pools(self):
        if self.cache == "e4m3":
            return self.k.numpy(), self.v.numpy(), self.ke.numpy(), self.ve.numpy()
        return self.k.double().numpy(), self.v.double().numpy(), None, None

    def attention(self, q, window=0):
        k, v, ke, ve = self.oracle_pools()
        return G.attention(q.double().numpy(), k, v, ke, ve, self.row_start, self.kv_len, self.pages, self.page,
                           self.max_rows, window)

    def largest_score_sum(self, q):
        """max over rows, heads and slots of sum |q_i k_i| / sqrt(hd), from above (norms)."""
        k, _, ke, _ = self.oracle_pools()
        x = G.widen(k, ke) if ke is not None else k
        x = np.where(self.used.numpy()[:, None, :, None], x, 0.0)
        x = np.where(np.isfinite(x), x, 0.0)
        kn = np.sqrt((x ** 2).sum(-1)).max()
        qd = q.double().numpy()
        return float(np.sqrt((qd ** 2).sum(-1)).max() * kn / math.sqrt(self.hd))


def attention_bound(s: Setup, q, ref, spread, few_rows: bool):
    """How far a result may be from 64 bits, element by element, from the arithmetic.

    With u = 2^-24: a score is a sum of hd products in fp32, off by at most (hd + 2) u S with S >= sum |q_i k_i| /
    sqrt(hd) >= |s|; its scaling into the exponent, the maximum's and their difference add 4 u S; exp2 and expf are off
    by 2 u relative (the hardware's is 1 ulp). So a weight is off by d = 2 ((hd + 6) u S + 4 u) relative, before and
    after normalisation by at most twice that. Sums over n slots add n u, the joins of four waves and of the splits and
    the division 64 u. A weight rounded to bf16 is off by 2^-8 (in numerator and denominator: twice), as hi and lo by
    2^-16. All of it counts against sum w |v|; the stored result adds half a step of itself."""
    u = 2.0 ** -24
    S = s.largest_score_sum(q)
    n = max(s.kv_len + [1])
    d = 2 * ((s.hd + 6) * u * S + 4 * u)
    rel = 2 * d + 2 * n * u + 64 * u
    if s.dtype == "bf16":
        rel += 2 * 2.0 ** -16 if few_rows else 2 * 2.0 ** -8 * (1 + 2.0 ** -7)
    return rel * spread + HALF[s.dtype] * np.abs(ref) * (1 + rel) + 1e-30
