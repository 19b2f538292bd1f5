"""Embedding, norms and the head's losses without a GPU: refusals of the C entry points and of the binding, workspace
sizes. Nothing here launches a kernel."""
import pytest
import torch

import paper_2607_21291_amd as P

FAKE = 0x100000  # never dereferenced
OK_BUT_NO_GPU = 5
BIG = 1 << 45
without_gpu = pytest.mark.skipif(torch.cuda.is_available(), reason="placeholder pointers")


def _embed(tokens=FAKE, table=FAKE, dtype=P.BF16, n=10, V=100, d=64, scale=1.0, out=FAKE):
    return P.lib().dsf_embed_forward(tokens, table, dtype, n, V, d, scale, out, None)


def _embed_grad(tokens=FAKE, dy=FAKE, dtype=P.BF16, n=10, V=100, d=64, scale=1.0, acc=0, dtable=FAKE, kind=P.F32, ws=FAKE,
                nbytes=BIG):
    return P.lib().dsf_embed_backward(tokens, dy, dtype, n, V, d, scale, acc, dtable, kind, ws, nbytes, None)


def _norm(x=FAKE, w=FAKE, b=FAKE, dtype=P.BF16, n=10, d=64, eps=1e-5, rms=0, out=FAKE):
    return P.lib().dsf_norm_forward(x, w, b, dtype, n, d, eps, rms, out, None)


def _norm_grad(x=FAKE, dy=FAKE, w=FAKE, add=None, dtype=P.BF16, n=10, d=64, eps=1e-5, rms=0, dx=FAKE, dw=FAKE, db=FAKE,
               ws=FAKE, nbytes=BIG):
    return P.lib().dsf_norm_backward(x, dy, w, add, dtype, n, d, eps, rms, dx, dw, db, ws, nbytes, None)


def _ce(h=FAKE, w=FAKE, dtype=P.BF16, n=10, d=64, V=100, targets=FAKE, weight=None, scale=1.0, mean=0, loss=FAKE,
        total=FAKE, dh=FAKE, dw=FAKE, kind=P.BF16, ws=FAKE, nbytes=BIG):
    return P.lib().dsf_head_cross_entropy(h, w, dtype, n, d, V, targets, weight, scale, mean, loss, total, dh, dw, kind, ws,
                                          nbytes, None)


def _distill(h=FAKE, w=FAKE, dtype=P.BF16, n=10, d=64, V=100, top=FAKE, value=FAKE, k=8, T=1.0, weight=None, scale=1.0,
             mean=0, loss=FAKE, total=FAKE, dh=FAKE, dw=FAKE, kind=P.BF16, ws=FAKE, nbytes=BIG):
    return P.lib().dsf_head_distill(h, w, dtype, n, d, V, top, value, k, T, weight, scale, mean, loss, total, dh, dw, kind,
                                    ws, nbytes, None)


NAN, INF = float("nan"), float("inf")
BAD = {
    _embed: [(dict(dtype=2), 2), (dict(n=-1), 1), (dict(n=1 << 30), 1), (dict(V=0), 1), (dict(d=0), 2), (dict(d=20), 2),
             (dict(d=16392), 2), (dict(tokens=None), 1), (dict(table=None), 1), (dict(out=None), 1),
             (dict(table=FAKE + 8), 1), (dict(out=FAKE + 4), 1), (dict(tokens=FAKE + 2), 1)],
    _embed_grad: [(dict(dtype=7), 2), (dict(n=-1), 1), (dict(V=-3), 1), (dict(d=12), 2), (dict(dtable=None), 1),
                  (dict(dy=None), 1), (dict(tokens=None), 1), (dict(dy=FAKE + 8), 1), (dict(dtable=FAKE + 8), 1),
                  (dict(kind=P.BF16, dtype=P.F32), 2), (dict(kind=5), 2), (dict(ws=None), 3), (dict(ws=FAKE + 64), 1),
                  (dict(nbytes=100), 3)],
    _norm: [(dict(dtype=3), 2), (dict(n=-1), 1), (dict(d=4), 2), (dict(d=20000), 2), (dict(eps=-1.0), 1),
            (dict(eps=NAN), 1), (dict(eps=INF), 1), (dict(x=None), 1), (dict(w=None), 1), (dict(out=None), 1),
            (dict(b=FAKE + 2), 1), (dict(x=FAKE + 8), 1)],
    _norm_grad: [(dict(dtype=3), 2), (dict(n=-1), 1), (dict(d=4), 2), (dict(eps=-1.0), 1), (dict(x=None), 1),
                 (dict(dy=None), 1), (dict(w=None), 1), (dict(dx=None, dw=None, db=None), 1), (dict(rms=1), 1),
                 (dict(add=FAKE + 4), 1), (dict(dw=FAKE + 8), 1), (dict(ws=None), 3), (dict(nbytes=16), 3),
                 (dict(ws=FAKE + 16), 1)],
    _ce: [(dict(dtype=2), 2), (dict(n=-1), 1), (dict(n=(1 << 24) + 1), 1), (dict(d=100), 2), (dict(d=16400), 2),
          (dict(V=0), 2), (dict(V=(1 << 21) + 1), 2), (dict(h=None), 1), (dict(w=None), 1), (dict(targets=None), 1),
          (dict(h=FAKE + 8), 1), (dict(dh=FAKE + 8), 1), (dict(dw=FAKE + 2), 1), (dict(targets=FAKE + 1), 1),
          (dict(weight=FAKE + 2), 1), (dict(scale=NAN), 1), (dict(scale=INF), 1), (dict(kind=2), 2),
          (dict(kind=P.BF16, dtype=P.F32), 2), (dict(loss=None, total=None, dh=None, dw=None), 1), (dict(ws=None), 3),
          (dict(ws=FAKE + 128), 1), (dict(nbytes=4096), 3)],
    _distill: [(dict(k=0), 1), (dict(k=-1), 2), (dict(k=1025), 2), (dict(T=0.0), 1), (dict(T=-1.0), 1), (dict(T=NAN), 1),
               (dict(T=INF), 1), (dict(T=1e-7), 1), (dict(T=2e6), 1), (dict(top=None), 1), (dict(value=None), 1), (dict(value=FAKE + 2), 1), (dict(h=None), 1),
               (dict(nbytes=4096), 3), (dict(dtype=9), 2)],
}


@pytest.mark.parametrize("fn,kw,code", [(f, kw, code) for f, rows in BAD.items() for kw, code in rows])
def test_bad_arguments_are_refused(fn, kw, code):
    assert fn(**kw) == code and P.last_error()


@without_gpu
@pytest.mark.parametrize("fn", list(BAD))
def test_good_arguments_reach_the_device_check(fn):
    assert fn() == OK_BUT_NO_GPU


def test_empty_calls_need_no_gpu():
    assert _embed(n=0, tokens=None, table=None, out=None) == 0
    assert _embed_grad(n=0, acc=1, tokens=None, dy=None) == 0
    assert _norm(n=0, x=None, w=None, out=None, b=None) == 0
    assert _norm_grad(n=0, x=None, dy=None, w=None, dw=None, db=None) == 0
    assert _ce(n=0, h=None, w=None, targets=None, total=None, dw=None, ws=None, nbytes=0) == 0
    assert _distill(n=0, h=None, w=None, top=None, value=None, total=None, dw=None, ws=None, nbytes=0) == 0
    # a tensor without elements has no address: its output is not told from none
    none = dict(dh=None, dw=None, loss=None, total=None, ws=None, nbytes=0)
    assert _ce(n=0, h=None, w=None, targets=None, **none) == 0 and _distill(n=0, h=None, top=None, value=None, **none) == 0
    assert _norm_grad(n=0, x=None, dy=None, dx=None, dw=None, db=None) == 0


def test_workspace_sizes():
    assert P.embed_backward_workspace_size(0, 64, 100) > 0 and P.embed_backward_workspace_size(-1, 64, 100) == 0
    assert P.norm_backward_workspace_size(10, 12) == 0 and P.norm_backward_workspace_size(10, 16) > 0
    assert P.head_workspace_size(P.BF16, 10, 64, 0) == 0 and P.head_workspace_size(P.BF16, 10, 64, 100, top=2000) == 0
    assert P.head_workspace_size(P.E4M3, 10, 64, 100) == 0
    # never the logits of a call at once: 16 bits for each of as many rows as fit 4 GiB
    n, d, V = 1 << 17, 896, 151936
    size = P.head_workspace_size(P.BF16, n, d, V)
    assert 0 < size < (4 << 30) + 4 * V * d + 2 * n * d + (1 << 30) < 2 * n * V
    assert P.head_workspace_size(P.BF16, n, d, V, gradients=False) < size
    # enough for the call without gradients
    for args in [(100, 64, 1003), (5000, 896, 151936), (1, 8, 1)]:
        for dt in (P.F32, P.BF16):
            assert P.head_workspace_size(dt, *args, gradients=False) <= P.head_workspace_size(dt, *args)


def test_binding_checks_shapes_and_types():
    bf, i32 = torch.bfloat16, torch.int32
    tok, table, out = torch.zeros(4, dtype=i32), torch.zeros(9, 16, dtype=bf), torch.zeros(4, 16, dtype=bf)
    for args in [(tok.long(), table, out), (tok, table, out[:3]), (tok, table, out.float()), (tok, table[:, ::2], out),
                 (tok, table.double(), out), (tok, table[0], out), (tok, table, torch.zeros(4, 32, dtype=bf)[:, ::2]),
                 (tok, table, out)]:  # the last: not on a GPU
        with pytest.raises(ValueError):
            P.embed_forward(*args)
    with pytest.raises(ValueError):
        P.embed_backward(tok, out, table.half())
    with pytest.raises(ValueError):
        P.embed_backward(tok, out.float(), table)
    x, w = torch.zeros(4, 16), torch.ones(16)
    for kw in [dict(w=w[:8]), dict(b=w.double()), dict(out=x.t().contiguous()), dict()]:
        with pytest.raises(ValueError):
            P.norm_forward(**{"x": x, "w": w, "out": x, **kw})
    with pytest.raises(ValueError):
        P.norm_backward(x, x, w, x, dw=w.bfloat16())
    h, t = torch.zeros(4, 16, dtype=bf), torch.zeros(4, dtype=i32)
    for kw in [dict(targets=t[:3]), dict(targets=t.long()), dict(w=table.float()), dict(dw=table.half()),
               dict(total=torch.zeros(3)), dict(row_weight=torch.zeros(4, dtype=torch.float64)), dict(dh=h.float()), dict()]:
        with pytest.raises(ValueError):
            P.head_cross_entropy(**{"h": h, "w": table, "targets": t, **kw})
    with pytest.raises(ValueError):
        P.head_distill(h, table, torch.zeros(4, 3, dtype=i32), torch.zeros(4, 2))
