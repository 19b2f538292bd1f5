"""A training step's calls one after another: tokens, embedding, a routed layer, final norm, head loss; and back through
the norm's adjoint, the layer's backward, and the embedding's gradient, added to the head's (one table for both). The
whole step against 64 bits, which take the layer's kept positions as given, with the layer's tolerances (2e-2 of an
output's largest value, tests of the layer's backward); the ends alone, captured and replayed."""
import numpy as np
import pytest
import torch

import paper_2607_21291_amd as P
import synthetic as S
from ends_util import f64, rand
from gpu_util import TOL, announce, desc_dict, make_desc, rel_inf, workload, workspace
from oracle import adadsf_oracle as O
from oracle import ends_oracle as E

pytestmark = pytest.mark.gpu

V = 701


def _head(kind, h, table, data, **out):
    if kind == "ce":
        P.head_cross_entropy(h, table, data[0], mean=True, **out)
    else:
        P.head_distill(h, table, data[0], data[1], temperature=2.0, mean=True, **out)


def _data(kind, B, T, seed):
    g = torch.Generator().manual_seed(seed)
    tok = torch.randint(0, V, (B, T), generator=g).int()
    tok[1, T - 20:] = -1  # padding
    if kind == "ce":
        t = torch.roll(tok, -1, 1)
        t[:, -1] = -100
        t[0, :30] = -100  # a prompt
        return tok, (t.contiguous(),)
    top = torch.randint(0, V, (B, T, 8), generator=g).int()
    top[1, T - 20:] = -1
    return tok, (top, torch.randn(B, T, 8, generator=g) * 2)


@pytest.mark.parametrize("name", ["neox_bf16_small", "qwen_bf16_small"])
@pytest.mark.parametrize("kind", ["ce", "distill"])
def test_step(dev, name, kind):
    w = workload(name)
    B, T, d = w.batch, w.seq, w.d_model
    rms = w.block == S.QWEN
    W, table = S.layer_weights(w, 0), rand((V, d), "bf16", 3, 1.5 / d ** 0.5)
    gain, bias = rand((d,), "bf16", 4, 0.1, 1.0), None if rms else rand((d,), "bf16", 5, 0.1)
    tok, data = _data(kind, B, T, 7)
    scale = float(d) ** 0.5
    k = T // 2
    g = torch.Generator().manual_seed(1)
    idx = torch.stack([torch.randperm(T, generator=g)[:k].sort().values for _ in range(B)]).int()
    to = lambda t: None if t is None else t.to(dev)  # noqa: E731
    td, tokd, gd, bd, idd = to(table), to(tok), to(gain), to(bias), to(idx)
    dl, desc = P.DeviceLayer(W, dev), make_desc(w)
    announce(f"training step {name} {kind}")
    x0 = torch.empty(B, T, d, dtype=torch.bfloat16, device=dev)
    P.embed_forward(tokd, td, x0, scale=scale)
    y = x0.clone()
    P.sparse_block_forward(desc, dl.weights, y, k, workspace(w, B, T, k, dev), idx_in=idd)
    h = torch.empty_like(y)
    P.norm_forward(y, gd, h, b=bd, eps=w.norm_eps, rms=rms)
    dh, dtable, total = torch.empty_like(h), torch.empty(V, d, device=dev), torch.empty(2, device=dev)
    loss = torch.empty(B, T, device=dev)
    _head(kind, h, td, [to(t) for t in data], row_loss=loss, total=total, dh=dh, dw=dtable)
    dy, dgain = torch.empty_like(h), torch.empty(d, device=dev)
    dbias = None if rms else torch.empty(d, device=dev)
    P.norm_backward(y, dh, gd, dy, dw=dgain, db=dbias, eps=w.norm_eps, rms=rms)
    dx = torch.empty_like(x0)
    grads = {n: None for n in P.GRAD_FIELDS}
    grads["w_down"] = torch.empty(d, w.d_ff, device=dev)
    P.sparse_block_backward(desc, dl.weights, x0, dy, idd, dx, grads,
                            torch.empty(P.backward_workspace_size(desc, P.BF16, B, T, k), dtype=torch.uint8, device=dev))
    P.embed_backward(tokd, dx, dtable, scale=scale, accumulate=True)
    torch.cuda.synchronize()

    tn, tab = tok.numpy(), f64(table)
    rx = E.embed(tn, tab, scale)
    ry = O.routed_layer(desc_dict(w), W, rx, k, idx=idx.numpy().astype(np.int64))["y"]
    rh = E.norm(ry, f64(gain), f64(bias), w.norm_eps, rms).reshape(B * T, d)
    if kind == "ce":
        ref = E.cross_entropy(rh, tab, data[0].numpy().ravel(), mean=True)
    else:
        ref = E.distill(rh, tab, data[0].numpy().reshape(B * T, -1), data[1].numpy().reshape(B * T, -1), temperature=2.0,
                        mean=True)
    rdy, rdg, rdb = E.norm_grad(ry, ref["dh"].reshape(B, T, d), f64(gain), w.norm_eps, rms)
    back = O.routed_layer_backward(desc_dict(w), W, rx, rdy, idx.numpy().astype(np.int64))
    rdt = E.embed_grad(tn, back["dx"], V, scale, ref["dw"])[0]
    tol = TOL["bf16"]
    errs = {"loss": rel_inf(f64(loss).ravel(), ref["loss"]), "total": rel_inf(f64(total), ref["total"]),
            "dtable": rel_inf(f64(dtable), rdt), "dgain": rel_inf(f64(dgain), rdg), "dx": rel_inf(f64(dx), back["dx"]),
            "w_down": rel_inf(f64(grads["w_down"]), back["grads"]["w_down"])}
    if not rms:
        # the terms of a bias's gradient nearly cancel (a class's p and q over the rows), so that the layer's tolerance, of
        # the largest value, says nothing of it: N terms within tol max|dh| each are N tol max|dh| off together, many
        # times the sum itself. Against the terms that the step has, the bound of the norm's own tests: one rounding
        # for each addition of fp32 (rows in turn, 256 + 16 partial sums).
        terms = f64(dh).reshape(B * T, d)
        bound = (B * T / 1024 + 1 + 4096 / 16 + 16 + 4) * 2.0 ** -24 * np.abs(terms).sum(0)
        assert (np.abs(f64(dbias) - terms.sum(0)) <= bound).all()
        assert np.abs(f64(dbias) - rdb).max() <= B * T * tol * np.abs(ref["dh"]).max()
    print("[errors] " + " ".join(f"{n}={e:.1e}" for n, e in errs.items()), flush=True)
    for n, e in errs.items():
        assert e < tol, (n, e)


@pytest.mark.parametrize("kind", ["ce", "distill"])
def test_ends_captured(dev, kind):
    """Everything but the layer in one graph, on new tokens each replay, against the calls themselves, bit by bit."""
    B, T, d = 2, 150, 264
    table, gain = rand((V, d), "bf16", 3, 1.5 / d ** 0.5).to(dev), rand((d,), "bf16", 4, 0.1, 1.0).to(dev)
    sets = [_data(kind, B, T, s) for s in range(3)]
    n = B * T
    sizes = [P.head_workspace_size(P.BF16, n, d, V, top=8 if kind == "distill" else 0),
             P.norm_backward_workspace_size(n, d), P.embed_backward_workspace_size(n, d, V)]
    ws = [torch.empty(s, dtype=torch.uint8, device=dev) for s in sizes]
    tok, data = sets[0][0].to(dev), [t.to(dev) for t in sets[0][1]]

    def step(tok, data, ws):
        x, h, dh, dx = (torch.empty(B, T, d, dtype=torch.bfloat16, device=dev) for _ in range(4))
        dtable, dgain, total = torch.empty(V, d, device=dev), torch.empty(d, device=dev), torch.empty(2, device=dev)
        P.embed_forward(tok, table, x, scale=4.0)
        P.norm_forward(x, gain, h, rms=True)
        _head(kind, h, table, data, total=total, dh=dh, dw=dtable, workspace=ws[0])
        P.norm_backward(x, dh, gain, dx, dw=dgain, rms=True, workspace=ws[1])
        P.embed_backward(tok, dx, dtable, scale=4.0, accumulate=True, workspace=ws[2])
        return dtable, dgain, total

    eager = [step(t.to(dev), [x.to(dev) for x in more], [None] * 3) for t, more in sets]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    announce(f"ends captured {kind}")
    with torch.cuda.graph(graph):
        got = step(tok, data, ws)
    for _ in range(2):
        for (t, more), want in zip(sets, eager):
            tok.copy_(t)
            for a, b in zip(data, more):
                a.copy_(b)
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(got, want))
