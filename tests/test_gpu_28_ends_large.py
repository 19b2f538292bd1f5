"""Sizes whose offsets, or numbers of work items, pass 32 bits: embedding, norms, head losses. References in 64 bits on the
GPU, some rows at a time."""
import numpy as np
import pytest
import torch

import paper_2607_21291_amd as P
from ends_util import HALF, U
from gpu_util import announce

pytestmark = [pytest.mark.gpu, pytest.mark.slow]


def test_lookup_of_many_tokens(dev):
    n, V, d = (1 << 25) + 3, 50304, 128
    tok = torch.randint(-1, V, (n,), device=dev, dtype=torch.int32)
    table = torch.randn(V, d, device=dev).bfloat16()
    out = torch.empty(n, d, dtype=torch.bfloat16, device=dev)
    announce("embed, 8.6 GB")
    P.embed_forward(tok, table, out)
    for a in range(0, n, 1 << 23):
        t = tok[a:a + (1 << 23)].long()
        want = table[t.clamp(min=0)] * (t >= 0)[:, None]
        assert torch.equal(out[a:a + (1 << 23)], want)


def test_gradient_of_many_tokens(dev):
    n, V, d = (1 << 26) + 5, 1000, 8
    tok = torch.randint(-1, V + 1, (n,), device=dev, dtype=torch.int32)
    tok[: n // 8] = 7
    dy = torch.randn(n, d, device=dev, dtype=torch.bfloat16)
    got = torch.empty(V, d, device=dev)
    announce("embed gradient, 2^26 tokens")
    P.embed_backward(tok, dy, got)
    torch.cuda.synchronize()
    # sums on the CPU: additions of millions of rows to one place take the GPU's atomics minutes
    want, mag = np.zeros((V + 2, d)), np.zeros((V + 2, d))
    count = np.zeros(V + 2)
    for a in range(0, n, 1 << 24):
        t, y = tok[a:a + (1 << 24)].cpu().numpy() + 1, dy[a:a + (1 << 24)].t().float().cpu().numpy()
        count += np.bincount(t, minlength=V + 2)
        for c in range(d):
            want[:, c] += np.bincount(t, weights=y[c], minlength=V + 2)
            mag[:, c] += np.bincount(t, weights=np.abs(y[c]), minlength=V + 2)
    # pieces of 32 positions, then the pieces one after another
    bound = (32 + count[1:V + 1] / 32 + 4)[:, None] * U * mag[1:V + 1]
    assert (np.abs(got.double().cpu().numpy() - want[1:V + 1]) <= bound + 1e-30).all()


@pytest.mark.parametrize("rms", [False, True])
def test_norms_of_many_rows(dev, rms):
    n, d = (1 << 21) + 1, 2056  # 4.3e9 elements
    x = torch.randn(n, d, device=dev, dtype=torch.bfloat16)
    w = torch.randn(d, device=dev).bfloat16()
    dy = torch.randn(n, d, device=dev, dtype=torch.bfloat16)
    out = torch.empty_like(x)
    announce(f"norms, 8.6 GB a tensor, {rms}")
    P.norm_forward(x, w, out, rms=rms)
    dx, dw = torch.empty_like(x), torch.empty(d, device=dev)
    P.norm_backward(x, dy, w, dx, dw=dw, rms=rms)
    want_dw, mag = torch.zeros(d, dtype=torch.float64, device=dev), torch.zeros(d, dtype=torch.float64, device=dev)
    eps = float(np.float32(1e-5))
    for a in range(0, n, 1 << 17):
        X, Y = x[a:a + (1 << 17)].double(), dy[a:a + (1 << 17)].double()
        m = 0.0 if rms else X.mean(1, keepdim=True)
        r = (((X - m) ** 2).mean(1, keepdim=True) + eps) ** -0.5
        xh = (X - m) * r
        y = xh * w.double()
        # fp32 steps: 200 u of values below 40 and of what they are sums of (the norms' own tests derive less)
        assert ((out[a:a + (1 << 17)].double() - y).abs() <= 1.01 * HALF["bf16"] * y.abs() + 200 * U * 40).all()
        g = Y * w.double()
        want = r * (g - (0.0 if rms else g.mean(1, keepdim=True)) - xh * (g * xh).mean(1, keepdim=True))
        assert ((dx[a:a + (1 << 17)].double() - want).abs() <= 1.01 * HALF["bf16"] * want.abs() + 200 * U * 200).all()
        want_dw += (Y * xh).sum(0)
        mag += (Y * xh).abs().sum(0)
    # 2049 rows a workgroup, 1024 partial sums; xh off by 60 u
    assert ((dw.double() - want_dw).abs() <= (2049 + 1024 / 16 + 20 + 60) * U * mag).all()


def test_long_lists_of_many_rows(dev):
    n, k, V, d, T = 300001, 1024, 64, 8, 2.0
    h, w = torch.randn(n, d, device=dev).bfloat16(), torch.randn(V, d, device=dev).bfloat16()
    top = torch.randint(-1, V, (n, k), device=dev, dtype=torch.int32)
    value = torch.randn(n, k, device=dev)
    loss, total = torch.empty(n, device=dev), torch.empty(2, device=dev)
    announce("distill, 3e8 entries")
    P.head_distill(h, w, top, value, temperature=T, row_loss=loss, total=total)
    for a in list(range(0, n, 60000)):
        logp = torch.log_softmax(h[a:a + 2000].double() @ w.double().t() / T, 1)
        t = top[a:a + 2000].long()
        q = torch.softmax(torch.where(t >= 0, value[a:a + 2000].double() / T, -torch.inf), 1)
        want = T * T * (torch.special.xlogy(q, q) - q * logp.gather(1, t.clamp(min=0))).sum(1)
        # ends_util.head_bounds: 152 u of |z| + |lse| + 1 < 40, 104 u of |sum q log q| + 1 < 9, logits off by 100 u
        assert ((loss[a:a + 2000].double() - want).abs() <= T * T * (152 * 40 + 104 * 9 + 2 * 100 * 40) * U).all()
    # (a class that a list names again makes a loss that can be below 0) one rounding of a 64-bit sum
    assert (total[0].double() - loss.double().sum()).abs() <= 2 * U * loss.double().sum().abs() and total[1] == n


def test_head_of_more_than_4_gib(dev):
    n, d, V = 70, 1032, 1 << 21
    w = torch.empty(V, d, dtype=torch.bfloat16, device=dev)
    for a in range(0, V, 1 << 18):
        w[a:a + (1 << 18)] = (torch.randn(1 << 18, d, device=dev) * (2.5 / d ** 0.5)).bfloat16()
    h = torch.randn(n, d, device=dev).bfloat16()
    t = torch.randint(0, V, (n,), device=dev, dtype=torch.int32)
    t[0], t[1] = V - 1, V - 2
    loss, dh, dw = torch.empty(n, device=dev), torch.empty_like(h), torch.empty_like(w)
    announce("cross entropy, W of 4.3 GB")
    P.head_cross_entropy(h, w, t, row_loss=loss, dh=dh, dw=dw)
    H = h.double()
    z = torch.cat([H @ w[a:a + (1 << 18)].double().t() for a in range(0, V, 1 << 18)], 1)
    logp = torch.log_softmax(z, 1)
    assert (loss.double() + logp.gather(1, t.long()[:, None])[:, 0]).abs().max() < 2e-4  # logits off by some 1e-5
    dz = logp.exp_()
    dz[torch.arange(n, device=dev), t.long()] -= 1.0
    e, half = 1.1 * HALF["bf16"], HALF["bf16"]  # dz's rounding, its code and logits
    want, size = torch.zeros(n, d, dtype=torch.float64, device=dev), torch.zeros(n, d, dtype=torch.float64, device=dev)
    for a in range(0, V, 1 << 18):
        W, q = w[a:a + (1 << 18)].double(), dz[:, a:a + (1 << 18)]
        want += q @ W
        size += q.abs() @ W.abs()
        g, b = q.t() @ H, q.abs().t() @ H.abs()
        assert ((dw[a:a + (1 << 18)].double() - g).abs() <= e * b + 1.01 * half * g.abs() + 1e-30).all()
    assert ((dh.double() - want).abs() <= e * size + 1.01 * half * want.abs()).all()
