"""The head's losses and gradients against 64 bits: cross entropy and distillation from top logits."""
import numpy as np
import pytest
import torch

import paper_2607_21291_amd as P
from ends_util import DT, HALF, close, f64, head_bounds, rand
from gpu_util import announce
from oracle import ends_oracle as E

pytestmark = pytest.mark.gpu

NAN = float("nan")
SIZES = [(1, 8, 1), (1, 64, 7), (3, 8, 300), (5, 72, 257), (17, 1536, 100), (130, 128, 1003), (300, 200, 515),
         (257, 768, 1300), (513, 264, 511), (1, 896, 5000), (700, 64, 40)]


def _inputs(n, d, V, dtype, seed=0):
    h, w = rand((n, d), dtype, seed), rand((V, d), dtype, seed + 1, 2.5 / d ** 0.5)
    return h, w


def _run(dev, call, h, w, *lists, grads=True, dw_type=None, **kw):
    n, d = h.shape
    out = {"row_loss": torch.full((n,), NAN, device=dev), "total": torch.full((2,), NAN, device=dev)}
    if grads:
        out["dh"] = torch.full((n, d), NAN, dtype=h.dtype, device=dev)
        out["dw"] = torch.full(tuple(w.shape), NAN, dtype=dw_type or w.dtype, device=dev)
    call(h.to(dev), w.to(dev), *[t.to(dev) for t in lists], **out, **kw)
    torch.cuda.synchronize()
    return out


def _check(out, ref, h, w, dtype, dw_type, lists=None):
    ref["lists"] = lists
    H, W = np.nan_to_num(f64(h)), f64(w)
    half_w = HALF["f32" if dw_type == torch.float32 else dtype]
    loss, dh, dw = head_bounds(ref, H, W, dtype, HALF[dtype], half_w)
    close(out["row_loss"], ref["loss"], loss, "loss")
    wt = np.abs(ref["weight"] * ref["live"])
    tb = np.array([(wt * loss).sum() + HALF["f32"] * abs(ref["total"][0]), HALF["f32"] * abs(ref["total"][1])])
    close(out["total"], ref["total"], tb + 1e-38, "total")
    if "dh" in out:
        close(out["dh"], ref["dh"], dh, "dh")
        close(out["dw"], ref["dw"], dw, "dw")
        assert out["dh"].cpu()[~torch.from_numpy(ref["live"])].eq(0).all()


def _targets(n, V, masked, seed):
    g = torch.Generator().manual_seed(seed)
    t = torch.randint(0, V, (n,), generator=g)
    t[torch.rand(n, generator=g) < masked] = -100
    if masked and n > 4:
        t[n // 2] = V  # no class either
    return t.int()


@pytest.mark.parametrize("n,d,V", SIZES)
@pytest.mark.parametrize("dtype,dw_type", [("bf16", torch.bfloat16), ("bf16", torch.float32), ("f32", torch.float32)])
@pytest.mark.parametrize("masked,weighted,mean", [(0.0, False, True), (0.4, True, False), (0.4, False, True)])
def test_cross_entropy(dev, n, d, V, dtype, dw_type, masked, weighted, mean):
    h, w = _inputs(n, d, V, dtype, n)
    t = _targets(n, V, masked, 5)
    weight = (torch.rand(n, generator=torch.Generator().manual_seed(6)) - 0.2).float() if weighted else None
    if weighted and n > 2:
        weight[1] = 0.0
    dead = (t < 0) | (t >= V) | ((weight == 0) if weighted else torch.zeros(n, dtype=torch.bool))
    h[dead] = NAN  # rows that take no part have no effect
    announce(f"cross entropy {n} {d} {V} {dtype} {dw_type} {masked} {weighted} {mean}")
    kw = dict(row_weight=None if weight is None else weight.to(dev), grad_scale=0.7, mean=mean)
    out = _run(dev, P.head_cross_entropy, h, w, t, dw_type=dw_type, **kw)
    ref = E.cross_entropy(np.nan_to_num(f64(h)), f64(w), t.numpy(), weight=None if weight is None else weight.numpy(),
                          grad_scale=float(np.float32(0.7)), mean=mean)
    _check(out, ref, h, w, dtype, dw_type)
    alone = _run(dev, P.head_cross_entropy, h, w, t, grads=False, **kw)
    assert torch.equal(alone["row_loss"], out["row_loss"]) and torch.equal(alone["total"], out["total"])


@pytest.mark.parametrize("n,d,V", SIZES)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("k,T", [(1, 1.0), (5, 2.0), (64, 0.5), (130, 4.0)])
def test_distill(dev, n, d, V, dtype, k, T):
    h, w = _inputs(n, d, V, dtype, n + 50)
    g = torch.Generator().manual_seed(k)
    top = torch.randint(0, V, (n, k), generator=g)  # a class twice in some lists
    top[torch.rand(n, k, generator=g) < 0.2] = -1
    value = torch.randn(n, k, generator=g) * 3 + 5
    value[torch.rand(n, k, generator=g) < 0.1] = -float("inf")
    if n > 3:
        top[2] = V + 1
        value[3] = -float("inf")
    value[top < 0] = NAN  # of entries that are none
    live = ((top >= 0) & (top < V) & (value != -float("inf"))).any(1)
    h[~live] = NAN
    announce(f"distill {n} {d} {V} {dtype} {k} {T}")
    out = _run(dev, P.head_distill, h, w, top.int(), value, temperature=T, mean=True)
    ref = E.distill(np.nan_to_num(f64(h)), f64(w), top.numpy(), value.numpy(), temperature=T, mean=True)
    _check(out, ref, h, w, dtype, w.dtype, lists=k)


@pytest.mark.parametrize("n,d,V", [(33, 8, 65), (64, 136, 1000), (65, 72, 129), (100, 904, 3001), (128, 64, 64), (129, 64, 300), (250, 72, 999)])
@pytest.mark.parametrize("dw_type", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("masked", [0.0, 0.5])
def test_few_rows(dev, n, d, V, dw_type, masked):
    """dz has two terms up to 128 rows that take part: one large entry's rounding is not a row's error."""
    h, w = _inputs(n, d, V, "bf16", n)
    t = _targets(n, V, masked, 8)
    h[(t < 0) | (t >= V)] = NAN
    announce(f"few rows {n} {d} {V} {dw_type} {masked}")
    weight = 0.5 + torch.rand(n, generator=torch.Generator().manual_seed(n))
    out = _run(dev, P.head_cross_entropy, h, w, t, dw_type=dw_type, mean=True, row_weight=weight.to(dev))
    ref = E.cross_entropy(np.nan_to_num(f64(h)), f64(w), t.numpy(), mean=True, weight=weight.numpy())
    _check(out, ref, h, w, "bf16", dw_type)
    teacher = torch.stack([t, t.roll(1)], 1).contiguous()
    value = torch.randn(n, 2, generator=torch.Generator().manual_seed(n))
    h = torch.nan_to_num(h)
    out = _run(dev, P.head_distill, h, w, teacher, value, temperature=2.0, dw_type=dw_type)
    _check(out, E.distill(f64(h), f64(w), teacher.numpy(), value.numpy(), temperature=2.0), h, w, "bf16", dw_type, lists=2)


@pytest.mark.parametrize("n", [1, 63, 64, 65, 130, 192, 193, 300, 321, 400])
@pytest.mark.parametrize("masked", [0.0, 0.4])
def test_few_rows_in_fp32(dev, n, masked):
    """Either side of the tiles' choices, by the rows that take part."""
    d, V = 136, 1400
    h, w = _inputs(n, d, V, "f32", n)
    t = _targets(n, V, masked, 8)
    h[(t < 0) | (t >= V)] = NAN
    announce(f"few rows, fp32 {n} {masked}")
    out = _run(dev, P.head_cross_entropy, h, w, t, mean=True)
    _check(out, E.cross_entropy(np.nan_to_num(f64(h)), f64(w), t.numpy(), mean=True), h, w, "f32", w.dtype)


def test_one_entry_at_temperature_one_is_cross_entropy(dev):
    h, w = _inputs(70, 128, 900, "bf16")
    t = _targets(70, 900, 0.2, 1)
    a = _run(dev, P.head_cross_entropy, h, w, t)
    b = _run(dev, P.head_distill, h, w, t[:, None].contiguous(), torch.randn(70, 1))
    assert torch.equal(a["dh"], b["dh"]) and torch.equal(a["dw"], b["dw"])
    assert torch.allclose(a["row_loss"], b["row_loss"], rtol=0, atol=1e-6)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_no_row_takes_part(dev, dtype):
    h, w = _inputs(40, 64, 333, dtype)
    h[:] = NAN
    for t, weight in [(torch.full((40,), -100), None), (torch.arange(40), torch.zeros(40))]:
        out = _run(dev, P.head_cross_entropy, h, w, t.int(), row_weight=None if weight is None else weight.to(dev),
                   mean=True)
        assert all(v.eq(0).all() for v in out.values())
    out = _run(dev, P.head_distill, h, w, torch.full((40, 3), -1).int(), torch.zeros(40, 3), mean=True)
    assert all(v.eq(0).all() for v in out.values())
    out = _run(dev, P.head_cross_entropy, h[:0], w, torch.zeros(0, dtype=torch.int32), mean=True)
    assert out["total"].eq(0).all() and out["dw"].eq(0).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_far_logits(dev, dtype):
    """Rows that are sure, rows of equal logits, logits far below a row's maximum."""
    d, V = 64, 1000
    w = torch.zeros(V, d)
    w[:, 0] = torch.linspace(-1, 1, V)
    w[:, 1] = (torch.arange(V) == 17).float()
    h = torch.zeros(6, d)
    h[1, 0], h[2, 0], h[3, 1], h[4, 1], h[5, 0] = 300.0, -300.0, 100.0, -80.0, 3.0e4
    h, w = h.to(DT[dtype]), w.to(DT[dtype])
    t = torch.tensor([5, 999, 999, 17, 17, 0], dtype=torch.int32)
    announce(f"far logits {dtype}")
    out = _run(dev, P.head_cross_entropy, h, w, t)
    _check(out, E.cross_entropy(f64(h), f64(w), t.numpy()), h, w, dtype, w.dtype)


def test_a_bad_row_spoils_its_own_results(dev):
    h, w = _inputs(300, 128, 700, "bf16")
    t = _targets(300, 700, 0.0, 3)
    good = _run(dev, P.head_cross_entropy, h, w, t)
    h[7], h[200, 3] = NAN, float("inf")
    bad = _run(dev, P.head_cross_entropy, h, w, t)
    rest = torch.tensor([i for i in range(300) if i not in (7, 200)])
    assert torch.equal(bad["row_loss"].cpu()[rest], good["row_loss"].cpu()[rest])
    assert torch.equal(bad["dh"].cpu()[rest], good["dh"].cpu()[rest])
    assert bad["row_loss"][7].isnan() and bad["dh"][7].isnan().all() and bad["dw"].isnan().any()


@pytest.mark.parametrize("dtype,n,V", [("bf16", 1200, 1 << 21), ("f32", 600, (1 << 21) - 5), ("bf16", 3200, 700001)])
@pytest.mark.parametrize("dw_type", ["same", "f32"])
def test_rows_in_pieces(dev, dtype, n, V, dw_type):
    """More rows than fit one piece of the workspace. The reference is taken on the GPU in 64 bits, half the rows at a
    time; dz's rounding (and p's code) dominate: 1.1 of its half step."""
    d = 16
    h, w = _inputs(n, d, V, dtype)
    t = _targets(n, V, 0.1, 9)
    announce(f"pieces {dtype} {n} {V} {dw_type}")
    out = _run(dev, P.head_cross_entropy, h, w, t, dw_type=torch.float32 if dw_type == "f32" else w.dtype, mean=True)
    H, W, tt = h.to(dev).double(), w.to(dev).double(), t.to(dev).long()
    live = (tt >= 0) & (tt < V)
    scale = 1.0 / float(live.sum())
    dw, bw = torch.zeros_like(W), torch.zeros_like(W)
    e = 1.1 * HALF[dtype] + (2e-5 if dtype == "f32" else 0.0)  # fp32: logits off by some 1e-6
    for r in torch.arange(n, device=dev).split(200):
        r = r[live[r]]
        logp = torch.log_softmax(H[r] @ W.t(), 1)
        loss = -logp.gather(1, tt[r][:, None])[:, 0]
        assert (out["row_loss"][r].double() - loss).abs().max() < 2e-5
        dz = logp.exp_()
        dz[torch.arange(len(r), device=dev), tt[r]] -= 1.0
        want, size = scale * (dz @ W), scale * (dz.abs() @ W.abs())
        dw += scale * (dz.t() @ H[r])
        dz.abs_()
        bw += scale * (dz.t() @ H[r].abs())
        half = HALF[dtype]
        assert ((out["dh"][r].double() - want).abs() <= e * size + 1.01 * half * want.abs()).all()
        del logp, dz
    half = HALF["f32" if dw_type == "f32" else dtype]
    assert ((out["dw"].double() - dw).abs() <= e * bw + 1.01 * half * dw.abs() + 1e-30).all()


def test_equal_bits_streams_and_replays(dev):
    n, d, V = 600, 256, 2000
    w = _inputs(1, d, V, "bf16")[1].to(dev)
    hs = [_inputs(n, d, V, "bf16", s)[0].to(dev) for s in range(3)]
    ts = [_targets(n, V, m, s).to(dev) for s, m in enumerate((0.0, 0.9, 0.5))]

    def call(h, t, **kw):
        o = [torch.empty(n, device=dev), torch.empty(2, device=dev), torch.empty_like(h), torch.empty_like(w)]
        P.head_cross_entropy(h, w, t, row_loss=o[0], total=o[1], dh=o[2], dw=o[3], mean=True, **kw)
        return o

    eager = [call(h, t) for h, t in zip(hs, ts)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for i in range(6):
        got = call(hs[i % 3], ts[i % 3], stream=streams[i % 2])
        streams[i % 2].synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, eager[i % 3]))
    h, t = hs[0].clone(), ts[0].clone()
    ws = torch.empty(P.head_workspace_size(P.BF16, n, d, V), dtype=torch.uint8, device=dev)
    g = torch.cuda.CUDAGraph()
    announce("cross entropy captured")
    with torch.cuda.graph(g):
        got = call(h, t, workspace=ws)
    for _ in range(2):
        for a, b, want in zip(hs, ts, eager):
            h.copy_(a)
            t.copy_(b)
            g.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(x, y) for x, y in zip(got, want))


def test_differences(dev):
    """Gradients against central differences of the losses themselves (fp32). The loss of 4 rows is off by some 1e-5,
    the step is 0.05, the third derivatives of a loss are below 1: 1e-5 / 0.05 + 0.05^2 / 6 < 1e-3 a row."""
    n, d, V, k, T = 4, 16, 50, 6, 1.5
    h, w = _inputs(n, d, V, "f32")
    g = torch.Generator().manual_seed(1)
    top, value = torch.randint(0, V, (n, k), generator=g).int(), torch.randn(n, k, generator=g)
    t = _targets(n, V, 0.0, 2)
    for call, lists, kw in [(P.head_cross_entropy, (t,), {}), (P.head_distill, (top, value), {"temperature": T})]:
        out = _run(dev, call, h, w, *lists, **kw)
        for seed in range(3):
            dh, dw = rand((n, d), "f32", 30 + seed, 0.25), rand((V, d), "f32", 40 + seed, 0.05)
            lo, hi = (f64(_run(dev, call, h + s * dh, w + s * dw, *lists, grads=False, **kw)["row_loss"]).sum()
                      for s in (-0.05, 0.05))
            want = (f64(out["dh"]) * f64(dh)).sum() + (f64(out["dw"]) * f64(dw)).sum()
            assert abs((hi - lo) / 0.1 - want) < n * 4e-3


@pytest.mark.parametrize("T", [0.5, 1.0, 3.0])
def test_teacher_logits_of_the_lowest_value(dev, T):
    """Masks of the type's lowest value are logits: alone in a list they share it, beside others they weigh nothing."""
    n, d, V, k = 4, 64, 300, 5
    h, w = _inputs(n, d, V, "f32")
    top = torch.arange(n * k).view(n, k).int()
    value = torch.full((n, k), torch.finfo(torch.float32).min)
    value[1, 2], value[2, :2], value[3, 1:] = 4.0, torch.tensor([3.0e38, 1.0]), -float("inf")
    announce(f"lowest logits {T}")
    out = _run(dev, P.head_distill, h, w, top, value, temperature=T)
    ref = E.distill(f64(h), f64(w), top.numpy(), value.numpy(), temperature=T)
    assert ref["live"].all()
    _check(out, ref, h, w, "f32", w.dtype, lists=k)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,d,V", [(37, 72, 257), (300, 128, 1003)])
def test_workspaces_of_any_contents(dev, dtype, n, d, V):
    """What a workspace holds before a call (here every bit set, NaN in both types) has no effect."""
    h, w = (x.to(dev) for x in _inputs(n, d, V, dtype))
    t = _targets(n, V, 0.3, 4).to(dev)
    top = torch.stack([t, t.roll(1), t.roll(2)], 1).contiguous()
    value = torch.randn(n, 3, device=dev)
    for call, lists, k in [(P.head_cross_entropy, (t,), 0), (P.head_distill, (top, value), 3)]:
        ws = torch.zeros(P.head_workspace_size(P.F32 if dtype == "f32" else P.BF16, n, d, V, top=k), dtype=torch.uint8,
                         device=dev)
        got = []
        for fill in (0, 255):
            ws.fill_(fill)
            got.append(_run(dev, call, h, w, *lists, workspace=ws, mean=True))
        assert all(torch.equal(got[0][x], got[1][x]) and got[0][x].isfinite().all() for x in got[0])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,d,V", [(37, 72, 257), (300, 128, 1003)])
def test_dh_in_the_place_of_h(dev, dtype, n, d, V):
    h, w = (x.to(dev) for x in _inputs(n, d, V, dtype))
    t = _targets(n, V, 0.3, 4).to(dev)
    want = _run(dev, P.head_cross_entropy, h, w, t, mean=True)
    total, row_loss, dw, dh = torch.empty(2, device=dev), torch.empty(n, device=dev), torch.empty_like(w), h.clone()
    announce(f"dh in the place of h {dtype} {n} {d} {V}")
    P.head_cross_entropy(dh, w, t, row_loss=row_loss, total=total, dh=dh, dw=dw, mean=True)
    got = {"row_loss": row_loss, "total": total, "dh": dh, "dw": dw}
    assert all(torch.equal(got[x], want[x]) for x in want)
