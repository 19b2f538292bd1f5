"""Pins of the 64-bit plain forms of embedding, norms and the head's losses: torch's own forms and autograd in float64."""
import numpy as np
import pytest
import torch

from oracle import ends_oracle as E

F = torch.nn.functional


def _t(a):
    return torch.tensor(a, dtype=torch.float64, requires_grad=True)


def test_embedding_and_its_gradient():
    rng = np.random.default_rng(0)
    tok = rng.integers(-2, 9, (5, 4))
    table, dy = rng.normal(size=(7, 3)), rng.normal(size=(5, 4, 3))
    ok = (tok >= 0) & (tok < 7)
    t = _t(table)
    out = F.embedding(torch.tensor(np.where(ok, tok, 0)), t) * 2.5 * torch.tensor(ok[..., None])
    out.backward(torch.tensor(dy))
    assert np.allclose(E.embed(tok, table, 2.5), out.detach().numpy(), atol=1e-14)
    got, mag, count = E.embed_grad(tok, dy, 7, 2.5)
    assert np.allclose(got, t.grad.numpy(), atol=1e-13) and (mag >= np.abs(got) - 1e-12).all() and count.sum() == ok.sum()


@pytest.mark.parametrize("rms", [False, True])
def test_norms(rms):
    rng = np.random.default_rng(1)
    x, dy, w, b = rng.normal(size=(6, 10)) + 1, rng.normal(size=(6, 10)), rng.normal(size=10), rng.normal(size=10)
    X, W, B = _t(x), _t(w), _t(b)
    y = F.rms_norm(X, (10,), W, 1e-3) if rms else F.layer_norm(X, (10,), W, B, 1e-3)
    y.backward(torch.tensor(dy))
    assert np.allclose(E.norm(x, w, None if rms else b, 1e-3, rms), y.detach().numpy(), atol=1e-13)
    dx, dw, db = E.norm_grad(x, dy, w, 1e-3, rms, add=dy)
    assert np.allclose(dx - dy, X.grad.numpy(), atol=1e-13) and np.allclose(dw, W.grad.numpy(), atol=1e-13)
    if not rms:
        assert np.allclose(db, B.grad.numpy(), atol=1e-13)


@pytest.mark.parametrize("mean", [False, True])
def test_cross_entropy(mean):
    rng = np.random.default_rng(2)
    h, w, t = rng.normal(size=(8, 5)), rng.normal(size=(11, 5)), rng.integers(0, 11, 8)
    t[3], weight = -100, rng.uniform(size=8)
    H, W = _t(h), _t(w)
    loss = F.cross_entropy(H @ W.t(), torch.tensor(t), reduction="none", ignore_index=-100)
    wt = torch.tensor(weight) * torch.tensor(t >= 0)
    (0.3 * (wt * loss).sum() / (wt.sum() if mean else 1.0)).backward()
    ref = E.cross_entropy(h, w, t, weight=weight, grad_scale=0.3, mean=mean)
    assert np.allclose(ref["loss"], loss.detach().numpy()) and np.allclose(ref["total"][1], wt.sum().item())
    assert np.allclose(ref["dh"], H.grad.numpy()) and np.allclose(ref["dw"], W.grad.numpy())


def test_distill():
    rng = np.random.default_rng(3)
    n, V, k, T = 6, 13, 4, 2.0
    h, w, v = rng.normal(size=(n, 5)), rng.normal(size=(V, 5)), rng.normal(size=(n, k))
    top = np.array([rng.permutation(V)[:k] for _ in range(n)])
    top[1, 2], v[2, 0], top[4] = -1, -np.inf, V
    top[5, 3] = top[5, 0]  # a class twice
    q = np.zeros((n, V))
    H, W = _t(h), _t(w)
    logp = F.log_softmax(H @ W.t() / T, 1)
    loss = []
    for i in range(n):
        ok = [j for j in range(k) if 0 <= top[i, j] < V and np.isfinite(v[i, j])]
        if not ok:
            loss.append(torch.zeros((), dtype=torch.float64))
            continue
        qi = torch.softmax(torch.tensor(v[i, ok]) / T, 0)
        loss.append(T * T * (qi * (qi.log() - logp[i, torch.tensor(top[i, ok])])).sum())
    loss = torch.stack(loss)
    loss.sum().backward()
    ref = E.distill(h, w, top, v, temperature=T)
    assert np.allclose(ref["loss"], loss.detach().numpy())
    assert np.allclose(ref["dh"], H.grad.numpy()) and np.allclose(ref["dw"], W.grad.numpy())
    assert not ref["live"][4] and ref["live"].sum() == n - 1
