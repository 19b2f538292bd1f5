"""The norm adjoint's sums over rows, to what their additions can lose. A workgroup adds its rows one after another, n over
the workgroups of them (up to 512 rows 256 workgroups, then one for two rows, 1024 at most); sixteen chains add the
workgroups' sums, and one the chains'. Each addition loses u of the magnitudes, each product and xh what norm_bounds says."""
import numpy as np
import pytest
import torch

import paper_2607_21291_amd as P
from ends_util import U, f64, norm_bounds, rand
from gpu_util import announce
from oracle import ends_oracle as E

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n,d", [(1, 64), (300, 72), (1023, 520), (5000, 264), (33000, 40)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rms", [False, True])
@pytest.mark.parametrize("same_sign", [False, True])
def test_sums_over_rows(dev, n, d, dtype, rms, same_sign):
    x, w = rand((n, d), dtype, n, 1.0, 0.5), rand((d,), dtype, 1, 0.2, 1.0)
    dy = rand((n, d), dtype, 2)
    if same_sign:
        dy = dy.abs()
    dw, db = torch.full((d,), float("nan"), device=dev), None if rms else torch.full((d,), float("nan"), device=dev)
    announce(f"norm sums {n} {d} {dtype} {rms} {same_sign}")
    P.norm_backward(x.to(dev), dy.to(dev), w.to(dev), torch.empty_like(x, device=dev), dw=dw, db=db, rms=rms)
    eps = float(np.float32(1e-5))
    X, Y = f64(x), f64(dy)
    _, want_dw, want_db = E.norm_grad(X, Y, f64(w), eps, rms)
    ex, _, xh, _ = norm_bounds(X, f64(w), None, eps, rms)
    wgs = min(n, 1024, max(256, (n + 1) // 2))
    chain = -(-n // wgs) + -(-wgs // 16) + 16 + 1
    assert (np.abs(f64(dw) - want_dw) <= (np.abs(Y) * ex).sum(0) + chain * U * np.abs(Y * xh).sum(0)).all()
    if db is not None:
        assert (np.abs(f64(db) - want_db) <= chain * U * np.abs(Y).sum(0)).all()
