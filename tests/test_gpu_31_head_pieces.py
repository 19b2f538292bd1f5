"""The head's losses for more rows than one piece of the workspace holds, in every form: cross entropy and distillation,
weights, totals, losses alone, three pieces (a middle one adds to a sum that another goes on with), later pieces without a
row, few enough rows for dz in two terms; and dh or dW alone. References in 64 bits on the GPU, some rows at a time.

Widths are small, logits off by some 1e-6: 2e-5 cover a loss (T^2 as much). dz is off by its rounding to dtype, its code
and its logits: 1.1 half steps of bf16; where at most 128 rows take part, by 1.1 of the code's (fp32: by 2e-5).

dh adds V / 2 products of two classes in fp32, which at 2^21 classes says more than dz: each addition rounds a sum of at most
`size`, the terms' magnitudes, by 2 u of it if all go one way, V u together; as roundings to nearest that know nothing of each
other, u / sqrt(3) each, they make sqrt(V / 2) u of `size` as a root of the mean square (an fp32 product of the library half
of that, the kernel a twentieth)."""
import numpy as np
import pytest
import torch

import paper_2607_21291_amd as P
from ends_util import CODE, HALF, U, rand
from gpu_util import announce

pytestmark = pytest.mark.gpu

BIGGEST = 1 << 21  # classes: 1024 rows a piece in bf16, 512 in fp32


def _case(n, d, V, dtype, masked, k, weighted, seed=0):
    h, w = rand((n, d), dtype, seed), rand((V, d), dtype, seed + 1, 2.5 / d ** 0.5)
    g = torch.Generator().manual_seed(seed + 2)
    dead = torch.rand(n, generator=g) < masked
    weight = torch.rand(n, generator=g) + 0.25 if weighted else None
    cls = torch.randint(0, V, (n, max(k, 1)), generator=g).int()
    cls[:, k // 2 + 1:][torch.rand(n, max(k - k // 2 - 1, 0) if k else 0, generator=g) < 0.3] = -1
    cls[dead] = V + 3
    h[dead] = float("nan")
    value = torch.randn(n, k, generator=g) * 2 if k else None
    return h, w, cls if k else cls[:, 0].contiguous(), value, weight, ~dead


def _call(dev, h, w, cls, value, weight, T, dw_type, want=("row_loss", "total", "dh", "dw")):
    n, V = len(h), len(w)
    out = {"row_loss": torch.full((n,), float("nan"), device=dev), "total": torch.full((2,), float("nan"), device=dev),
           "dh": torch.full_like(h, float("nan"), device=dev),
           "dw": torch.full(w.shape, float("nan"), dtype=dw_type, device=dev)}
    out = {x: out[x] for x in want}
    kw = dict(out, row_weight=None if weight is None else weight.to(dev), grad_scale=0.7, mean=True)
    if value is None:
        P.head_cross_entropy(h.to(dev), w.to(dev), cls.to(dev), **kw)
    else:
        P.head_distill(h.to(dev), w.to(dev), cls.to(dev), value.to(dev), temperature=T, **kw)
    torch.cuda.synchronize()
    return out


def _check(dev, out, h, w, cls, value, weight, live, T, dtype, rows=None):
    """rows: those whose losses are compared (all of them where gradients are)."""
    W = w.to(dev).double()
    wt = torch.ones(len(h), dtype=torch.float64) if weight is None else weight.double()
    wt = (wt * live).to(dev)
    wsum = float(wt.sum())
    two = dtype == "bf16" and int(live.sum()) <= 128
    e = 2e-5 if dtype == "f32" else 1.1 * (CODE if two else HALF["bf16"])
    scale = float(np.float32(0.7)) * T / wsum
    dw, bw = torch.zeros_like(W), torch.zeros_like(W)
    at = torch.nonzero(live)[:, 0] if rows is None else rows
    cd = cls.to(dev).long().view(len(h), -1)
    for r in at.to(dev).split(200):
        H = h[r.cpu()].to(dev).double()
        logp = torch.log_softmax(H @ W.t() / T, 1)
        ok = (cd[r] >= 0) & (cd[r] < len(w))
        idx = cd[r].where(ok, 0)
        if value is None:
            q = ok.double()
        else:
            q = torch.softmax(torch.where(ok, value[r.cpu()].to(dev).double() / T, -torch.inf), 1)
        loss = T * T * (torch.special.xlogy(q, q) - q * logp.gather(1, idx)).sum(1)
        assert (out["row_loss"][r].double() - loss).abs().max() <= 2e-5 * T * T
        if "dh" not in out:
            continue
        dz = logp.exp_().scatter_add_(1, idx, -q).mul_(wt[r][:, None])
        want, size = scale * (dz @ W), scale * (dz.abs() @ W.abs())
        err, chain = out["dh"][r].double() - want, 0.0
        if dtype == "f32":
            chain = (len(w) + 260) * U
            assert float((err / size).square().mean().sqrt()) <= (len(w) / 2) ** 0.5 * U + 2e-5
        assert (err.abs() <= (e + chain) * size + 1.01 * HALF[dtype] * want.abs() + 1e-30).all()
        dw += scale * (dz.t() @ H)
        bw += scale * (dz.abs_().t() @ H.abs())
        del logp, dz
    dead = torch.nonzero(~live)[:, 0].to(dev)
    assert out["row_loss"][dead].eq(0).all()
    # one rounding of a 64-bit sum of the losses themselves
    total = (wt * out["row_loss"].double()).sum()
    assert (out["total"][0].double() - total).abs() <= 2.0 ** -23 * total.abs()
    assert abs(float(out["total"][1]) - wsum) <= 2.0 ** -23 * wsum
    if "dw" in out:
        assert out["dh"][dead].eq(0).all()
        half = HALF["f32"] if out["dw"].dtype == torch.float32 else HALF["bf16"]
        assert ((out["dw"].double() - dw).abs() <= e * bw + 1.01 * half * dw.abs() + 1e-30).all()


@pytest.mark.parametrize("dtype,n,V,masked", [
    ("bf16", 2600, BIGGEST, 0.1),      # three pieces with rows
    ("bf16", 2600, BIGGEST - 9, 0.7),  # two without a row
    ("bf16", 2600, BIGGEST, 0.97),     # dz in two terms
    ("f32", 1200, BIGGEST, 0.1),       # three pieces
    ("f32", 1200, BIGGEST - 9, 0.8),   # two without a row
])
@pytest.mark.parametrize("k,T,weighted,dw_type", [(0, 1.0, True, "same"), (0, 1.0, False, "f32"), (6, 2.0, True, "same"),
                                                  (1, 0.5, False, "f32")])
def test_pieces(dev, dtype, n, V, masked, k, T, weighted, dw_type):
    h, w, cls, value, weight, live = _case(n, 8, V, dtype, masked, k, weighted)
    announce(f"pieces {dtype} {n} {V} {masked} {k} {T} {weighted} {dw_type}")
    out = _call(dev, h, w, cls, value, weight, T, torch.float32 if dw_type == "f32" else w.dtype)
    _check(dev, out, h, w, cls, value, weight, live, T, dtype)


@pytest.mark.parametrize("dtype,n", [("bf16", 66000), ("f32", 1200)])
@pytest.mark.parametrize("k", [0, 6])
def test_losses_alone_in_pieces(dev, dtype, n, k):
    """bf16 keeps no logits here: a piece is as many rows as its statistics allow, 65536 of 2^21 classes."""
    h, w, cls, value, weight, live = _case(n, 8, BIGGEST, dtype, 0.3, k, True)
    announce(f"losses alone in pieces {dtype} {n} {k}")
    out = _call(dev, h, w, cls, value, weight, 2.0 if k else 1.0, None, want=("row_loss", "total"))
    at = torch.nonzero(live)[:, 0]
    _check(dev, out, h, w, cls, value, weight, live, 2.0 if k else 1.0, dtype, rows=torch.cat([at[:150], at[-150:]]))


@pytest.mark.parametrize("dtype,n,d,V,masked", [("bf16", 300, 264, 1003, 0.2), ("bf16", 70, 264, 1003, 0.0), ("bf16", 1, 64, 5, 0.0),
                                                ("f32", 300, 264, 1003, 0.2), ("bf16", 2600, 8, BIGGEST, 0.1),
                                                ("f32", 1200, 8, BIGGEST, 0.7)])
@pytest.mark.parametrize("k", [0, 6])
def test_one_gradient_alone(dev, dtype, n, d, V, masked, k):
    """dh alone (a head that is not trained), dW alone, losses alone, no losses: the same bits as with everything."""
    h, w, cls, value, weight, live = _case(n, d, V, dtype, masked, k, True)
    announce(f"one gradient alone {dtype} {n} {d} {V} {k}")
    run = lambda *want: _call(dev, h, w, cls, value, weight, 2.0 if k else 1.0, w.dtype, want)  # noqa: E731
    every = run("row_loss", "total", "dh", "dw")
    assert all(t.isfinite().all() for t in every.values())
    for want in (("dh",), ("dw",), ("total", "dh"), ("row_loss", "dw"), ("dh", "dw"), ("total",), ("row_loss",)):
        got = run(*want)
        assert all(torch.equal(got[x], every[x]) for x in want), want


def test_pieces_bounded_by_partial_sums(dev):
    """Few classes of wide rows: 65536 rows of width 16384 are 4 GiB of dh's partial sums. Logits are sums below 10 of 528
    additions: some 1e-5 off, 1e-4 at most; dz by 1.1 of its half step, dW's own additions (n / 32, 2 u each) make it 1.2."""
    n, d, V = 66000, 16384, 6
    g = torch.Generator(device=dev).manual_seed(3)
    h = torch.randn(n, d, device=dev, dtype=torch.bfloat16, generator=g)
    w = (torch.randn(V, d, device=dev, generator=g) * (2.5 / d ** 0.5)).bfloat16()
    t = torch.randint(-1, V, (n,), device=dev, dtype=torch.int32, generator=g)
    assert P.head_workspace_size(P.BF16, n, d, V) < n * d * 2 + (5 << 30)
    loss, total, dh, dw = (torch.empty(x, device=dev, dtype=y) for x, y in (
        (n, torch.float32), (2, torch.float32), ((n, d), torch.bfloat16), ((V, d), torch.float32)))
    announce("pieces bounded by partial sums")
    P.head_cross_entropy(h, w, t, row_loss=loss, total=total, dh=dh, dw=dw, mean=True)
    W, e = w.double(), 1.2 * HALF["bf16"]
    want_dw, size_dw = torch.zeros_like(W), torch.zeros_like(W)
    live = t >= 0
    scale, sum_loss = 1.0 / float(live.sum()), 0.0
    for a in range(0, n, 4096):
        H, tt, ok = h[a:a + 4096].double(), t[a:a + 4096].long(), live[a:a + 4096]
        logp = torch.log_softmax(H @ W.t(), 1)
        want = -logp.gather(1, tt.clamp(min=0)[:, None])[:, 0] * ok
        assert (loss[a:a + 4096].double() - want).abs().max() <= 1e-4
        sum_loss += float(want.sum())
        dz = logp.exp().scatter_add_(1, tt.clamp(min=0)[:, None], -torch.ones_like(logp[:, :1])) * ok[:, None]
        want, size = scale * (dz @ W), scale * (dz.abs() @ W.abs())
        assert ((dh[a:a + 4096].double() - want).abs() <= e * size + 1.01 * HALF["bf16"] * want.abs() + 1e-30).all()
        want_dw += scale * (dz.t() @ H)
        size_dw += scale * (dz.abs().t() @ H.abs())
    assert ((dw.double() - want_dw).abs() <= e * size_dw).all()
    assert abs(float(total[0]) - sum_loss) <= 1e-4 * n and float(total[1]) == float(live.sum())
