"""Rows that are sure of their target: a loss and a gradient that are differences of nearly equal numbers. The target's
logit and the log-sum have to come from the same sums, or the difference is the rounding of a logit (1e-5 and more at 30)
instead of the rounding of 1.

With M the greatest logit of a row in units of log 2 and S = sum 2^(z - M), a target of probability near 1 has loss
ln 2 (M - z + log2 S). M - z is exact up to a rounding of itself; S is 2^(M - z) to 2 u (exp2 to a unit in the last place)
and takes the other classes' terms, below 2^-26 together, without any change; the logarithm of a value that near 1 is off
by 1.5 times as much, 3 u, and twice 2 u for the exponential in dz: 8 u cover a loss (at temperature 1) and p - 1."""
import numpy as np
import pytest
import torch

import paper_2607_21291_amd as P
from ends_util import HALF, U, f64, head_bounds, rand
from gpu_util import announce
from oracle import ends_oracle as E

pytestmark = pytest.mark.gpu

SURE = 8 * U


def _run(dev, call, h, w, *lists, **kw):
    out = {"row_loss": torch.empty(len(h), device=dev), "total": torch.empty(2, device=dev),
           "dh": torch.empty_like(h, device=dev), "dw": torch.empty(w.shape, device=dev)}
    call(h.to(dev), w.to(dev), *[t.to(dev) for t in lists], **out, **kw)
    torch.cuda.synchronize()
    return {k: f64(v) for k, v in out.items()}


def _rows(n, d, V, z, dtype, seed=0):
    """h, w, targets: each row's logit is about z at its target and about z / sqrt(d) in size elsewhere."""
    w = rand((V, d), "f32", seed + 1, d ** -0.5).to(torch.bfloat16).float()
    t = torch.randint(0, V, (n,), generator=torch.Generator().manual_seed(seed + 2))
    h = z * w[t] / (w[t] ** 2).sum(1, keepdim=True)
    h = h + 0.01 * rand((n, d), "f32", seed + 3)
    kind = torch.float32 if dtype == "f32" else torch.bfloat16
    return h.to(kind), w.to(kind), t.int()


def _check(out, ref, h, w, dtype, T, classes):
    """Against 64 bits: losses, and gradients as products of dz that is off by SURE at the targets. Elsewhere p, which the
    logits' own error, some percent of a factor of two at most, and codes change by less than a tenth; in bf16 a p below 2^-64
    of the greatest among its neighbours, which is at most 1, is 0, so p is off by at most 2^-64 there."""
    n, V = len(h), len(w)
    t = np.where(ref["live"], classes, 0)
    near = 1.0 - ref["p"][np.arange(n), t]
    assert (near < 2.0 ** -26).all()
    assert (out["row_loss"] >= 0).all(), out["row_loss"].min()
    assert (np.abs(out["row_loss"] - ref["loss"]) <= T * T * SURE + 0.1 * ref["loss"]).all(), \
        (np.abs(out["row_loss"] - ref["loss"]).max(), T * T * SURE)
    edz = 0.1 * ref["p"] + (2.0 ** -64 if dtype == "bf16" else 0.0)
    edz[np.arange(n), t] = SURE
    edz *= (np.abs(ref["weight"]) * ref["live"])[:, None]
    s, H, W = abs(ref["scale"]), f64(h), f64(w)
    dh, dw = s * edz @ np.abs(W) * 1.01, s * edz.T @ np.abs(H) * 1.01
    assert (np.abs(out["dh"] - ref["dh"]) <= dh + HALF[dtype] * (np.abs(ref["dh"]) + dh) + 1e-38).all(), "dh"
    assert (np.abs(out["dw"] - ref["dw"]) <= dw + 1e-38).all(), "dw"


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,d", [(1, 8), (5, 72), (130, 896), (300, 3584), (700, 264)])
def test_one_class(dev, dtype, n, d):
    """A head of one class: p is 1 whatever the logit."""
    h = rand((n, d), dtype, n, 30.0 * d ** -0.5)
    w = h[n // 2:n // 2 + 1] / 5
    t = torch.zeros(n, dtype=torch.int32)
    announce(f"one class {dtype} {n} {d}")
    out = _run(dev, P.head_cross_entropy, h, w, t)
    ref = E.cross_entropy(f64(h), f64(w), t.numpy())
    _check(out, ref, h, w, dtype, 1.0, t.numpy())
    out = _run(dev, P.head_distill, h, w, t[:, None].contiguous(), torch.randn(n, 1), temperature=3.0)
    ref = E.distill(f64(h), f64(w), t[:, None].numpy(), np.zeros((n, 1)), temperature=3.0)
    _check(out, ref, h, w, dtype, 3.0, t.numpy())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,d,V", [(64, 3584, 1003), (200, 3584, 1003), (517, 904, 777), (33, 328, 5000)])
@pytest.mark.parametrize("z", [45.0, 80.0])
def test_sure_rows(dev, dtype, n, d, V, z):
    h, w, t = _rows(n, d, V, z, dtype)
    announce(f"sure rows {dtype} {n} {d} {V} {z}")
    out = _run(dev, P.head_cross_entropy, h, w, t)
    _check(out, E.cross_entropy(f64(h), f64(w), t.numpy()), h, w, dtype, 1.0, t.numpy())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("k,T", [(1, 2.0), (7, 1.0), (16, 0.5), (40, 2.0), (130, 1.0)])
def test_sure_rows_of_a_sure_teacher(dev, dtype, k, T):
    """Lists whose weight lies on the student's own class, anywhere in the list; the others' e^-100 / T and less."""
    n, d, V = 90, 904, 1200
    h, w, t = _rows(n, d, V, 60.0 * T, dtype)
    g = torch.Generator().manual_seed(k)
    top = torch.randint(0, V, (n, k), generator=g).int()
    value = torch.full((n, k), -300.0)
    at = torch.randint(0, k, (n,), generator=g)
    top[top == t[:, None]] = -1
    top[torch.arange(n), at] = t
    value[torch.arange(n), at] = 4.0
    announce(f"sure teacher {dtype} {k} {T}")
    out = _run(dev, P.head_distill, h, w, top, value, temperature=T)
    _check(out, E.distill(f64(h), f64(w), top.numpy(), value.numpy(), temperature=T), h, w, dtype, T, t.numpy())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("z", [4.0, 9.0, 14.0, 22.0])
def test_half_sure_rows(dev, dtype, z):
    """Between: a loss log(1 + e), e the others' sum over the target's term, moves by (1 - p) times the logits' errors; the
    sums' and the logarithm's own rounding is head_bounds'."""
    n, d, V = 150, 3584, 1003
    h, w, t = _rows(n, d, V, z, dtype)
    announce(f"half sure rows {dtype} {z}")
    out = _run(dev, P.head_cross_entropy, h, w, t)
    ref = E.cross_entropy(f64(h), f64(w), t.numpy())
    ref["lists"] = None
    step = 32 if dtype == "bf16" else 2
    H, W = f64(h), f64(w)
    # a chain of d / step additions of sums of step, 2 u each, of what the products add up to in size; scaled: 4 u of z
    ez = (2 * (d / step + step) * U * (np.abs(H) @ np.abs(W).T) + 6 * U * np.abs(ref["z"])).max(1)
    near = 1.0 - ref["p"][np.arange(n), t.numpy()]
    L = V / 4096 + 64 if dtype == "bf16" else V / 1024 + 64
    bound = np.expm1(2 * ez) * near + (L + 8) * U * (1 + ref["loss"])
    assert (np.abs(out["row_loss"] - ref["loss"]) <= bound).all(), (np.abs(out["row_loss"] - ref["loss"]) / bound).max()
    _, dh, dw = head_bounds(ref, H, W, dtype, HALF[dtype], HALF["f32"])
    assert (np.abs(out["dh"] - ref["dh"]) <= dh).all() and (np.abs(out["dw"] - ref["dw"]) <= dw).all()
