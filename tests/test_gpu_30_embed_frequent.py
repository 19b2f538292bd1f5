"""The embedding's gradient for tokens that hold most of a batch: the error of a sum must not grow with how often its token
occurs. Pieces of 32 positions are fp32 sums (31 additions: 31 u of the magnitudes at most), eight pieces are added pairwise
(3 u), these in 64 bits; then one rounding to fp32, the scaling and the addition to what was there: 37 u, and the rounding of
the output."""
import numpy as np
import pytest
import torch

import paper_2607_21291_amd as P
from ends_util import DT, HALF, U, f64
from gpu_util import announce

pytestmark = pytest.mark.gpu


def _grad(tok, dy, V):
    """Sums by token and of the terms' magnitudes, in 64 bits."""
    t, y = tok.numpy().astype(np.int64) + 1, f64(dy)
    t[t > V] = 0
    pick = lambda a: np.stack([np.bincount(t, weights=a[:, c], minlength=V + 1)[1:] for c in range(a.shape[1])], 1)  # noqa: E731
    return pick(y), pick(np.abs(y))


@pytest.mark.parametrize("kind", ["positive", "equal", "signed"])
@pytest.mark.parametrize("dtype,out,add", [("bf16", "f32", False), ("f32", "f32", True), ("bf16", "bf16", True)])
@pytest.mark.parametrize("n,V,d,share", [(1 << 22, 700, 8, 1.0), (1 << 20, 5, 24, 0.5), (40007, 999, 520, 0.97)])
def test_frequent_tokens(dev, n, V, d, share, kind, dtype, out, add):
    g = torch.Generator().manual_seed(n)
    tok = torch.randint(-1, V + 1, (n,), generator=g).int()
    tok[torch.rand(n, generator=g) < share] = V - 2
    dy = torch.rand(n, d, generator=g)
    if kind == "equal":
        dy = torch.tensor([0.1, 0.7, 0.013, 3.3, 0.9, 1e-3, 0.23, 5.1]).repeat(d // 8).expand(n, d)
    elif kind == "signed":
        dy = dy * 2 - 1
    dy = dy.to(DT[dtype]).contiguous()
    start = torch.randn(V, d, generator=g).to(DT[out])
    got = start.to(dev) if add else torch.full((V, d), float("nan"), dtype=DT[out], device=dev)
    announce(f"frequent tokens {n} {V} {d} {share} {kind} {dtype} {out} {add}")
    P.embed_backward(tok.to(dev), dy.to(dev), got, scale=1.7, accumulate=add)
    torch.cuda.synchronize()
    s = float(np.float32(1.7))
    want, mag = (s * a for a in _grad(tok, dy, V))
    if add:
        want, mag = want + f64(start), mag + np.abs(f64(start))
    bound = 38 * U * mag
    err = np.abs(f64(got) - want)
    assert (err <= bound + HALF[out] * (np.abs(want) + bound) + 1e-38).all(), (err / (U * mag + 1e-300)).max()
