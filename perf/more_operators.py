"""The two ends of a training step around the layer stack, as programs call
them: the embedding lookup and its gradient, the final norm and its adjoint,
the head's cross entropy with its gradients (no logits are kept), and the same
for distillation from a teacher's top logits.

Widths and vocabularies are those of the package's workloads and benchmark.
Tokens are distributed by rank as in text (log-uniform over the vocabulary, so
that the commonest one takes several percent of the places). Hidden rows are
N(0, 1), as a final norm leaves them, turned towards the row of the head that
belongs to their target; the head's rows have a deviation that spreads logits
by 2.5, so that some rows are sure of their target and some are not. A part of
the rows has no target (prompts, padding).
"""
import math

import torch

own = False

# width, classes, norm with means and biases
MODELS = {
    "neox160m": (768, 50304, True),
    "neox14b": (2048, 50304, True),
    "qwen05b": (896, 151936, False),
    "qwen15b": (1536, 151936, False),
    "qwen7b": (3584, 151936, False),
    "tiny_neox": (128, 1003, True),
}
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "bf16": 2}


def _case(kind, model, dtype, rows, name=None, **more):
    c = {"kind": kind, "model": model, "dtype": dtype, "rows": rows, "classes": MODELS[model][1], "masked": 0.0,
         "add": False, "k": 0, "temperature": 1.0, "weighted": False}
    c.update(more)
    return dict(c, name=name) if name else c


def listed():
    return [
        # One token of each of a few decoding sequences: launch latency and little else.
        _case("embed", "neox160m", "bf16", 8, name="embed_tokens"),
        # The table's gradient for a training batch, written whole.
        _case("embed_grad", "qwen05b", "bf16", 16384, masked=0.1, name="embed_grad"),
        # A model whose head is its table: the gradient is added to the head's, in fp32.
        _case("embed_grad", "neox160m", "f32", 6001, masked=0.3, add=True, name="embed_grad_tied"),
        # The final norm of a decoding batch.
        _case("norm", "qwen7b", "bf16", 16, name="norm_tokens"),
        # The final norm of a training batch.
        _case("norm", "neox14b", "bf16", 8192, name="norm_train"),
        # Its adjoint and the gain's gradient, long sequences.
        _case("norm_grad", "qwen7b", "bf16", 32768, name="norm_grad"),
        # Scoring one text of a tokenizer whose size is no round number: losses only.
        _case("score", "neox160m", "bf16", 333, classes=50257, name="ce_score"),
        # A training batch of the smaller model, half prompt, half answer.
        _case("ce", "neox160m", "bf16", 16384, masked=0.5, name="ce_train"),
        # The largest: a training batch of the largest model.
        _case("ce", "qwen7b", "bf16", 8192, name="ce_train_large"),
        # Checking a small model in fp32.
        _case("ce", "neox160m", "f32", 700, masked=0.1, weighted=True, name="ce_f32"),
        # A short batch of stored teacher logits, 32 of a token.
        _case("distill", "qwen15b", "bf16", 250, k=32, temperature=1.0, weighted=True, name="distill_short"),
        # Distilling at a temperature from 64 logits of a token.
        _case("distill", "qwen05b", "bf16", 8192, masked=0.2, k=64, temperature=2.0, name="distill_train"),
    ]


def _active(case):
    return case["rows"] - int(case["rows"] * case["masked"])


def work(case):
    d, _, bias = MODELS[case["model"]]
    eb, n, V, a = BYTES[case["dtype"]], case["rows"], case["classes"], _active(case)
    kind = case["kind"]
    if kind == "embed":
        return {"bytes": n * 4 + 2 * n * d * eb, "flops": 0}
    if kind == "embed_grad":
        table = 2 * min(a, V) * d * 4 if case["add"] else V * d * eb
        return {"bytes": n * 4 + a * d * eb + table, "flops": 0}
    if kind == "norm":
        return {"bytes": 2 * n * d * eb + (2 if bias else 1) * d * eb, "flops": 0}
    if kind == "norm_grad":
        return {"bytes": 3 * n * d * eb + d * eb + (2 if bias else 1) * d * 4, "flops": 0}
    rows = n * 8 + n * case["k"] * 8
    if kind == "score":
        return {"bytes": rows + (a + V) * d * eb, "flops": 2 * a * V * d}
    return {"bytes": rows + (a + n + 2 * V) * d * eb, "flops": 6 * a * V * d}


def _cost(case):
    """About what the plain form of the case takes in seconds, to compare sizes."""
    w = work(case)
    return w["bytes"] / 1e12 + w["flops"] / 1e14


def draw(rng):
    """One more call of the same ranges."""
    def log(lo, hi):
        return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))

    limit = max(_cost(c) for c in listed())
    while True:
        kind = rng.choice(["embed", "embed_grad", "norm", "norm_grad", "score", "ce", "ce", "distill", "distill"])
        model, dtype = rng.choice(sorted(MODELS)), rng.choice(["bf16", "bf16", "bf16", "f32"])
        few = kind in ("ce", "distill", "score")
        rows = log(1, (20000 if dtype == "bf16" else 3000) if few else 40000)
        V = MODELS[model][1]
        more = {"classes": rng.choice([V, V - rng.randint(1, 500)])}
        if kind in ("embed_grad", "ce", "score", "distill"):
            more["masked"] = rng.choice([0.0, 0.1, 0.5, 0.9])
        if kind == "embed_grad":
            more["add"] = dtype == "f32" and rng.random() < 0.5
        if few:
            more["weighted"] = rng.random() < 0.3
        if kind == "distill":
            more.update(k=log(1, 128), temperature=rng.choice([0.5, 1.0, 2.0, 4.0]))
        c = _case(kind, model, dtype, rows, **more)
        if _cost(c) <= limit and rows * V <= 1.3e9:
            return c


def _tokens(n, V, gen, dev):
    """Ranks as in text: log-uniform, spread over the vocabulary by a fixed permutation."""
    u = torch.rand(n, generator=gen, device=dev, dtype=torch.float64)
    rank = (torch.exp(u * math.log(V + 1.0)) - 1.0).long().clamp_(0, V - 1)
    return (rank * 7919 + 13) % V


def _masked(case, gen, dev):
    m = torch.zeros(case["rows"], dtype=torch.bool, device=dev)
    m[torch.randperm(case["rows"], generator=gen, device=dev)[:case["rows"] - _active(case)]] = True
    return m


def prepare(case, seed):
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev).manual_seed(int(seed))
    d, _, bias = MODELS[case["model"]]
    dt, n, V, kind = DTYPES[case["dtype"]], case["rows"], case["classes"], case["kind"]
    normal = lambda *s: torch.randn(*s, generator=gen, device=dev)  # noqa: E731
    st = {"case": case, "scale": math.sqrt(d) if kind.startswith("embed") else 1.0}
    ws = 0
    if kind == "embed":
        st.update(tokens=_tokens(n, V, gen, dev).int(), table=(normal(V, d) * 0.02).to(dt),
                  out=torch.empty(n, d, dtype=dt, device=dev))
    elif kind == "embed_grad":
        tokens = _tokens(n, V, gen, dev)
        tokens[_masked(case, gen, dev)] = -1
        st.update(tokens=tokens.int(), dy=(normal(n, d) * 1e-2).to(dt))
        st["dtable"] = normal(V, d) * 1e-2 if case["add"] else torch.empty(V, d, dtype=dt, device=dev)
    elif kind in ("norm", "norm_grad"):
        # the residual stream: some columns are much larger than the others
        spread = torch.exp(normal(d) * 0.7)
        st.update(x=(normal(n, d) * spread + 0.3 * normal(d)).to(dt), w=(1 + 0.1 * normal(d)).to(dt),
                  b=(0.1 * normal(d)).to(dt) if bias else None, out=torch.empty(n, d, dtype=dt, device=dev))
        if kind == "norm_grad":
            st.update(dy=(normal(n, d) * 1e-2).to(dt), dw=torch.empty(d, device=dev),
                      db=torch.empty(d, device=dev) if bias else None)
    else:
        w = (normal(V, d) * (2.5 / math.sqrt(d))).to(dt)
        masked = _masked(case, gen, dev)
        if kind == "distill":
            # distinct classes: steps from a token; logits fall with their rank, some lists are shorter
            k = case["k"]
            first = _tokens(n, V, gen, dev)
            step = 1 + (torch.rand(n, generator=gen, device=dev) * (V // max(k, 2) - 1)).long()
            top = (first[:, None] + step[:, None] * torch.arange(k, device=dev)) % V
            value = 12.0 - 2.0 * torch.log1p(torch.arange(k, device=dev).float()) - normal(n, k).abs()
            short = torch.rand(n, generator=gen, device=dev) < 0.2
            top[:, k - k // 3:] = torch.where(short[:, None], -1, top[:, k - k // 3:])
            top[masked] = -1
            st.update(top=top.int(), value=value)
        else:
            first = _tokens(n, V, gen, dev)
            st["targets"] = torch.where(masked, -100, first).int()
        turn = 4.0 * torch.rand(n, 1, generator=gen, device=dev)
        h = normal(n, d)
        h += turn * torch.nn.functional.normalize(w[first].float(), dim=1)
        st.update(h=h.to(dt), w=w, weight=torch.rand(n, generator=gen, device=dev) if case["weighted"] else None,
                  loss=torch.empty(n, device=dev), total=torch.empty(2, device=dev))
        if kind != "score":
            st.update(dh=torch.empty(n, d, dtype=dt, device=dev), dw=torch.empty_like(w))
    if own:  # the workspace that a program keeps
        import paper_2607_21291_amd as P
        code = P.BF16 if case["dtype"] == "bf16" else P.F32
        if kind == "embed_grad":
            ws = P.embed_backward_workspace_size(n, d, V)
        elif kind == "norm_grad":
            ws = P.norm_backward_workspace_size(n, d)
        elif kind in ("ce", "score", "distill"):
            ws = P.head_workspace_size(code, n, d, V, top=case["k"], gradients=kind != "score")
        st["workspace"] = torch.empty(max(ws, 256), dtype=torch.uint8, device=dev)
    return st


def _own(st):
    import paper_2607_21291_amd as P
    case = st["case"]
    kind = case["kind"]
    if kind == "embed":
        P.embed_forward(st["tokens"], st["table"], st["out"], scale=st["scale"])
        return st["out"]
    if kind == "embed_grad":
        P.embed_backward(st["tokens"], st["dy"], st["dtable"], scale=st["scale"], accumulate=case["add"],
                         workspace=st["workspace"])
        return st["dtable"]
    if kind in ("norm", "norm_grad"):
        rms = st["b"] is None
        if kind == "norm":
            P.norm_forward(st["x"], st["w"], st["out"], b=st["b"], eps=1e-5, rms=rms)
            return st["out"]
        P.norm_backward(st["x"], st["dy"], st["w"], st["out"], dw=st["dw"], db=st["db"], eps=1e-5, rms=rms,
                        workspace=st["workspace"])
        return [st["out"], st["dw"], st["db"]]
    grads = {"dh": st["dh"], "dw": st["dw"]} if kind != "score" else {}
    args = dict(row_weight=st["weight"], row_loss=st["loss"], total=st["total"], mean=True,
                workspace=st["workspace"], **grads)
    if kind == "distill":
        P.head_distill(st["h"], st["w"], st["top"], st["value"], temperature=case["temperature"], **args)
    else:
        P.head_cross_entropy(st["h"], st["w"], st["targets"], **args)
    return [st["loss"], st["total"], *grads.values()]


def _plain_norm(st):
    x, w = st["x"].float(), st["w"].float()
    rms = st["b"] is None
    if not rms:
        x = x - x.mean(1, keepdim=True)
    rstd = 1.0 / torch.sqrt((x * x).mean(1, keepdim=True) + 1e-5)
    xh = x * rstd
    if st["case"]["kind"] == "norm":
        y = xh * w
        return (y if rms else y + st["b"].float()).to(st["x"].dtype)
    dy = st["dy"].float()
    g = dy * w
    dx = g - xh * (g * xh).mean(1, keepdim=True)
    if not rms:
        dx = dx - g.mean(1, keepdim=True)
    dw = (dy * xh).sum(0)
    return [(dx * rstd).to(st["x"].dtype), dw, None if rms else dy.sum(0)]


def run(st):
    if own:
        return _own(st)
    case = st["case"]
    kind, dt = case["kind"], DTYPES[case["dtype"]]
    if kind == "embed":
        return (st["table"][st["tokens"].long()].float() * st["scale"]).to(dt)
    if kind == "embed_grad":
        # places without a token go to a row behind the table
        V, d = st["dtable"].shape
        at = torch.where(st["tokens"] >= 0, st["tokens"].long(), V)
        got = torch.zeros(V + 1, d, device=at.device).index_add_(0, at, st["dy"].float() * st["scale"])[:V]
        return st["dtable"].add_(got) if case["add"] else got.to(dt)
    if kind in ("norm", "norm_grad"):
        return _plain_norm(st)
    h, w, T = st["h"].float(), st["w"].float(), case["temperature"]
    z = h @ w.t()
    if T != 1.0:
        z /= T
    top = z.max(1, keepdim=True).values
    lse = top + torch.log(torch.exp(z - top).sum(1, keepdim=True))
    if kind == "distill":
        at, there = st["top"].long().clamp(min=0), st["top"] >= 0
        q = torch.where(there, st["value"] / T, -math.inf)
        most = q.max(1, keepdim=True).values
        most = torch.where(torch.isfinite(most), most, 0.0)
        e = torch.exp(q - most)
        total = e.sum(1, keepdim=True)
        logq = q - most - torch.log(total)
        q = torch.where(there, e / total, 0.0)
        terms = torch.where(there, q * (logq - (z.gather(1, at) - lse)), 0.0)
        loss = T * T * terms.sum(1)
        active = there.any(1)
    else:
        at, active = st["targets"].long().clamp(min=0)[:, None], st["targets"] >= 0
        q = active.float()[:, None]
        loss = torch.where(active, (lse - z.gather(1, at))[:, 0], 0.0)
    weight = active.float() if st["weight"] is None else active * st["weight"]
    total = torch.stack([(weight.double() * loss).sum(), weight.double().sum()])
    if kind == "score":
        return [loss, total.float()]
    z -= lse
    dz = torch.exp_(z)
    dz.scatter_add_(1, at, -q)
    dz *= (weight * T / total[1]).float()[:, None]
    return [loss, total.float(), (dz @ w).to(dt), (dz.t() @ h).to(dt)]


def exact(case, seed):
    """From the definitions, in 64 bits, some rows at a time."""
    st = prepare(case, seed)
    kind = case["kind"]
    f = lambda t: t.to(torch.float64)  # noqa: E731
    if kind == "embed":
        return f(st["table"])[st["tokens"].long()] * st["scale"]
    if kind == "embed_grad":
        want = f(st["dtable"]) if case["add"] else torch.zeros(st["dtable"].shape, dtype=torch.float64,
                                                               device=st["dy"].device)
        keep = st["tokens"] >= 0
        return want.index_add(0, st["tokens"][keep].long(), f(st["dy"])[keep] * st["scale"])
    if kind in ("norm", "norm_grad"):
        n, d = st["x"].shape
        outs, dw, db = [], 0.0, 0.0
        for at in range(0, n, 4096):
            x = f(st["x"][at:at + 4096])
            mean = 0.0 if st["b"] is None else x.sum(1, keepdim=True) / d
            rstd = (((x - mean) ** 2).sum(1, keepdim=True) / d + 1e-5) ** -0.5
            xh = (x - mean) * rstd
            if kind == "norm":
                outs.append(xh * f(st["w"]) + (0.0 if st["b"] is None else f(st["b"])))
                continue
            dy = f(st["dy"][at:at + 4096])
            dw, db = dw + (dy * xh).sum(0), db + dy.sum(0)
            g = dy * f(st["w"])
            m1 = 0.0 if st["b"] is None else g.sum(1, keepdim=True) / d
            outs.append(rstd * (g - m1 - xh * ((g * xh).sum(1, keepdim=True) / d)))
        return torch.cat(outs) if kind == "norm" else [torch.cat(outs), dw, None if st["b"] is None else db]
    n, d = st["h"].shape
    V, T, dev = case["classes"], case["temperature"], st["h"].device
    w = f(st["w"])
    if kind == "distill":
        at = st["top"].long()
    else:
        at = st["targets"].long()[:, None]
    active = (at >= 0).any(1)
    weight = active.double() if st["weight"] is None else active * f(st["weight"])
    loss = torch.zeros(n, dtype=torch.float64, device=dev)
    dh, dw = torch.zeros(n, d, dtype=torch.float64, device=dev), torch.zeros_like(w)
    scale = weight / weight.sum()
    for r in torch.nonzero(active)[:, 0].split(1024):
        h = f(st["h"][r])
        logp = torch.log_softmax(h @ w.t() / T, 1)
        there, idx = at[r] >= 0, at[r].clamp(min=0)
        if kind == "distill":
            q = torch.softmax(torch.where(there, f(st["value"][r]) / T, -math.inf), 1)
        else:
            q = there.double()
        part = torch.where(there, torch.special.xlogy(q, q) - q * logp.gather(1, idx), 0.0)
        loss[r] = T * T * part.sum(1)
        if kind != "score":
            dz = logp.exp().scatter_add(1, idx, -q) * (T * scale[r])[:, None]
            dh[r] = dz @ w
            dw += dz.t() @ h
    total = torch.stack([(weight * loss).sum(), weight.sum()])
    return [loss, total] if kind == "score" else [loss, total, dh, dw]
