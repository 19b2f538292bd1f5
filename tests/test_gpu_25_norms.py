"""LayerNorm and RMSNorm of dense rows, and their adjoint, against 64 bits."""
import numpy as np
import pytest
import torch

import paper_2607_21291_amd as P
from ends_util import DT, HALF, U, close, f64, norm_bounds, rand
from gpu_util import announce
from oracle import ends_oracle as E

pytestmark = pytest.mark.gpu

SHAPES = [(1, 8), (1, 896), (3, 768), (16, 3584), (5, 2056), (2, 16384), (7, 8200), (1023, 64), (1024, 64), (1025, 520),
          (1500, 1024), (2050, 72), (1030, 3584), (4100, 1032), (2100, 1000)]


def _inputs(n, d, dtype, seed=0):
    g = torch.Generator().manual_seed(seed)
    x = (torch.randn(n, d, generator=g) * torch.exp(torch.randn(d, generator=g)) + torch.randn(n, 1, generator=g) * 3)
    return x.to(DT[dtype]), rand((d,), dtype, seed + 1, 0.2, 1.0), rand((d,), dtype, seed + 2, 0.3)


@pytest.mark.parametrize("n,d", SHAPES)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rms,bias", [(False, True), (False, False), (True, False), (True, True)])
def test_forward(dev, n, d, dtype, rms, bias):
    x, w, b = _inputs(n, d, dtype)
    b = b if bias else None
    out = torch.full_like(x, float("nan"), device=dev)
    announce(f"norm {n} {d} {dtype} {rms} {bias}")
    P.norm_forward(x.to(dev), w.to(dev), out, b=b.to(dev) if bias else None, eps=1e-5, rms=rms)
    eps = float(np.float32(1e-5))
    want = E.norm(f64(x), f64(w), f64(b), eps, rms)
    ex, _, xh, _ = norm_bounds(f64(x), f64(w), f64(b), eps, rms)
    bound = ex * np.abs(f64(w)) + 4 * U * (np.abs(xh * f64(w)) + (np.abs(f64(b)) if bias else 0.0))
    close(out, want, bound + HALF[dtype] * (np.abs(want) + bound) + 1e-38, "y")


@pytest.mark.parametrize("n,d", SHAPES)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rms", [False, True])
@pytest.mark.parametrize("wanted", ["all", "dx", "dw"])
def test_backward(dev, n, d, dtype, rms, wanted):
    x, w, _ = _inputs(n, d, dtype, 5)
    dy, add = rand((n, d), dtype, 8), rand((n, d), dtype, 9) if wanted == "all" else None
    nan = float("nan")
    dx = torch.full_like(x, nan, device=dev) if wanted != "dw" else None
    dw = torch.full((d,), nan, device=dev) if wanted != "dx" else None
    db = torch.full((d,), nan, device=dev) if wanted != "dx" and not rms else None
    announce(f"norm adjoint {n} {d} {dtype} {rms} {wanted}")
    P.norm_backward(x.to(dev), dy.to(dev), w.to(dev), dx, dw=dw, db=db, add=None if add is None else add.to(dev), eps=1e-6,
                    rms=rms)
    eps = float(np.float32(1e-6))
    X, Y, W = f64(x), f64(dy), f64(w)
    wx, ww, wb = E.norm_grad(X, Y, W, eps, rms, f64(add))
    ex, rr, xh, r = norm_bounds(X, W, None, eps, rms)
    g = Y * W
    L = d / 64 + 18
    mean = lambda a: a.mean(-1, keepdims=True)  # noqa: E731
    mg, mgx = (0.0 if rms else mean(g)), mean(g * xh)
    e_mg = 0.0 if rms else (L + 4) * U * mean(np.abs(g))
    e_mgx = (L + 6) * U * mean(np.abs(g * xh)) + mean(np.abs(g) * ex) + 2 * rr * np.abs(mgx)
    size = np.abs(g) + np.abs(mg) + np.abs(xh * mgx)
    ebx = r * (e_mg + np.abs(xh) * e_mgx + np.abs(mgx) * ex + (6 * U + rr) * size)
    if add is not None:
        ebx = ebx + 2 * U * np.abs(f64(add))
    if dx is not None:
        close(dx, wx, ebx + HALF[dtype] * (np.abs(wx) + ebx) + 1e-38, "dx")
    # a wave's rows one after another, then the partial sums in 16 chains, then 16
    chain = n / 1024 + 1 + 4096 / 16 + 16 + 4
    if dw is not None:
        close(dw, ww, (np.abs(Y) * ex).sum(0) + chain * U * np.abs(Y * xh).sum(0) + 1e-38, "dw")
    if db is not None:
        close(db, wb, chain * U * np.abs(Y).sum(0) + 1e-38, "db")


def test_in_place_no_rows_and_equal_bits(dev):
    x, w, b = (t.to(dev) for t in _inputs(2000, 904, "bf16"))
    dy = rand((2000, 904), "bf16", 1).to(dev)
    out = torch.empty_like(x)
    P.norm_forward(x, w, out, b=b)
    y = x.clone()
    P.norm_forward(y, w, y, b=b)
    assert torch.equal(y, out)
    res = []
    for _ in range(2):
        dx, dw, db = dy.clone(), torch.empty(904, device=dev), torch.empty(904, device=dev)
        P.norm_backward(x, dx if res else dy, w, dx, dw=dw, db=db)  # the second time in place of dy
        res.append((dx, dw, db))
    assert all(torch.equal(a, c) for a, c in zip(*res))
    dx, dw, db = x[:0], torch.full((904,), 7.0, device=dev), torch.full((904,), 7.0, device=dev)
    P.norm_backward(x[:0], dy[:0], w, dx, dw=dw, db=db)
    assert dw.eq(0).all() and db.eq(0).all()


def test_rows_do_not_touch_each_other(dev):
    x, w, b = _inputs(9, 640, "f32")
    x[3, 5], x[6] = float("nan"), float("inf")
    out = torch.empty(9, 640, device=dev)
    P.norm_forward(x.to(dev), w.to(dev), out, b=b.to(dev))
    bad = torch.tensor([3, 6])
    fine = torch.tensor([i for i in range(9) if i not in (3, 6)])
    assert out.cpu()[bad].isnan().all() and out.cpu()[fine].isfinite().all()


def test_replays(dev):
    n, d = 1300, 776
    xs = [_inputs(n, d, "bf16", s)[0].to(dev) for s in range(3)]
    dys = [rand((n, d), "bf16", 20 + s).to(dev) for s in range(3)]
    w = rand((d,), "bf16", 4, 0.1, 1.0).to(dev)
    x, dy = xs[0].clone(), dys[0].clone()
    ws = torch.empty(P.norm_backward_workspace_size(n, d), dtype=torch.uint8, device=dev)

    def call(x, dy, ws=None):
        out, dx = torch.empty_like(x), torch.empty_like(x)
        dw, db = torch.empty(d, device=dev), torch.empty(d, device=dev)
        P.norm_forward(x, w, out)
        P.norm_backward(x, dy, w, dx, dw=dw, db=db, workspace=ws)
        return out, dx, dw, db

    eager = [call(a, c) for a, c in zip(xs, dys)]
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = call(x, dy, ws)
    for _ in range(2):
        for a, c, want in zip(xs, dys, eager):
            x.copy_(a)
            dy.copy_(c)
            g.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(p, q) for p, q in zip(got, want))


@pytest.mark.parametrize("n,d", [(5, 2056), (1500, 1024), (2050, 72), (7, 8200), (3, 16384)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rms", [False, True])
def test_adjoint_in_place(dev, n, d, dtype, rms):
    """dx in the place of x, of dy or of add."""
    x, w, _ = (t.to(dev) for t in _inputs(n, d, dtype))
    dy, add = rand((n, d), dtype, 1).to(dev), rand((n, d), dtype, 2).to(dev)

    def call(x, dy, add, dx):
        dw = torch.empty(d, device=dev)
        P.norm_backward(x, dy, w, dx, dw=dw, add=add, rms=rms)
        return dx, dw

    announce(f"adjoint in place {n} {d} {dtype} {rms}")
    want = call(x, dy, add, torch.empty_like(x))
    for i in range(3):
        t = [x.clone(), dy.clone(), add.clone()]
        assert all(torch.equal(a, b) for a, b in zip(call(*t, t[i]), want))
