"""Embedding lookup and its gradient by sorted tokens against 64-bit sums."""
import numpy as np
import pytest
import torch

import paper_2607_21291_amd as P
from ends_util import DT, HALF, U, close, f64, rand
from gpu_util import announce
from oracle import ends_oracle as E

pytestmark = pytest.mark.gpu


def _tokens(n, V, kind, seed):
    g = torch.Generator().manual_seed(seed)
    if kind == "same":
        return torch.full((n,), V // 2, dtype=torch.int32)
    if kind == "none":
        return torch.full((n,), -1, dtype=torch.int32)
    t = torch.randint(0, V, (n,), generator=g)
    if kind == "skew":  # a third of the places hold two tokens, some hold none
        u = torch.rand(n, generator=g)
        t = torch.where(u < 0.2, V - 1, torch.where(u < 0.35, 0, torch.where(u < 0.45, -100, t)))
        t = torch.where(u > 0.97, V + 5, t)
    return t.int()


SIZES = [(1, 1, 8), (1, 300, 768), (8, 256, 896), (63, 257, 24), (64, 1003, 128), (65, 5, 520), (1000, 700, 1032),
         (4099, 50000, 64), (777, 3, 2048)]


@pytest.mark.parametrize("n,V,d", SIZES)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("scale", [1.0, 27.7])
def test_lookup(dev, n, V, d, dtype, scale):
    tok, table = _tokens(n, V, "skew", n), rand((V, d), dtype, 1)
    out = torch.full((n, d), float("nan"), dtype=DT[dtype], device=dev)
    announce(f"embed {n} {V} {d} {dtype} {scale}")
    P.embed_forward(tok.to(dev), table.to(dev), out, scale=scale)
    ok = (tok >= 0) & (tok < V)
    want = (table[tok.clamp(0, V - 1).long()].float() * np.float32(scale)).to(DT[dtype]) * ok[:, None]
    assert torch.equal(out.cpu().float() + 0.0, want.float() + 0.0)


def test_lookup_copies_bits_and_takes_batches(dev):
    table = torch.tensor([[float("nan"), float("inf"), -0.0, 1.0] * 2, [2.0] * 8], dtype=torch.bfloat16)
    tok = torch.tensor([[0, 1], [1, 0]], dtype=torch.int32)
    out = torch.empty(2, 2, 8, dtype=torch.bfloat16, device=dev)
    P.embed_forward(tok.to(dev), table.to(dev), out)
    assert torch.equal(out.cpu().view(torch.int16), table.view(torch.int16)[tok.long()])


@pytest.mark.parametrize("n,V,d", SIZES)
@pytest.mark.parametrize("kind", ["even", "skew", "same", "none"])
@pytest.mark.parametrize("dtype,out,add", [("bf16", "bf16", False), ("bf16", "f32", False), ("f32", "f32", False),
                                           ("bf16", "bf16", True), ("f32", "f32", True)])
def test_gradient(dev, n, V, d, kind, dtype, out, add):
    tok, dy = _tokens(n, V, kind, n + 1), rand((n, d), dtype, 2)
    dy[(tok < 0) | (tok >= V)] = float("nan")  # no effect
    start = rand((V, d), out, 3)
    got = start.to(dev) if add else torch.full((V, d), float("nan"), dtype=DT[out], device=dev)
    announce(f"embed gradient {n} {V} {d} {kind} {dtype} {out} {add}")
    P.embed_backward(tok.to(dev), dy.to(dev), got, scale=3.3, accumulate=add)
    scale = float(np.float32(3.3))
    want, mag, count = E.embed_grad(tok.numpy(), np.nan_to_num(f64(dy)), V, scale, f64(start) if add else None)
    # count additions, the scaling, the addition to what was there
    bound = (count[:, None] + 3) * U * mag
    close(got, want, bound + HALF[out] * (np.abs(want) + bound) + 1e-38, "dtable")
    if add:
        assert torch.equal(got.cpu()[count == 0], start[count == 0])


def test_gradient_equals_itself_and_survives_replays(dev):
    n, V, d = 3000, 999, 264
    toks = [_tokens(n, V, k, 7).to(dev) for k in ("skew", "same", "even")]
    dys = [rand((n, d), "bf16", 10 + i).to(dev) for i in range(3)]
    tok, dy = toks[0].clone(), dys[0].clone()
    ws = torch.empty(P.embed_backward_workspace_size(n, d, V), dtype=torch.uint8, device=dev)
    out = torch.empty(V, d, dtype=torch.bfloat16, device=dev)
    eager = []
    for t, y in zip(toks, dys):
        o = torch.empty_like(out)
        P.embed_backward(t, y, o, scale=0.5)
        eager.append(o)
    g = torch.cuda.CUDAGraph()
    announce("embed gradient captured")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        P.embed_backward(tok, dy, out, scale=0.5, workspace=ws)
    torch.cuda.current_stream().wait_stream(s)
    with torch.cuda.graph(g):
        P.embed_backward(tok, dy, out, scale=0.5, workspace=ws)
    for turn in range(2):
        for t, y, want in zip(toks, dys, eager):
            tok.copy_(t)
            dy.copy_(y)
            out.fill_(float("nan"))
            g.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, want)


def test_two_streams_with_workspaces_of_their_own(dev):
    n, V, d = 2048, 4000, 512
    tok, dy = _tokens(n, V, "skew", 3).to(dev), rand((n, d), "bf16", 4).to(dev)
    want = torch.empty(V, d, device=dev)
    P.embed_backward(tok, dy, want)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = [torch.empty(V, d, device=dev) for _ in range(6)]
    for i, o in enumerate(outs):
        P.embed_backward(tok, dy, o, stream=streams[i % 2])
    torch.cuda.synchronize()
    assert all(torch.equal(o, want) for o in outs)
