"""The paged key/value cache's operators, as programs call them: writing new
tokens' keys and values into pages (8-bit codes among them), reading them
back, and attention of each sequence's new tokens over its pages.

A batch holds B sequences. Sequence b brings the rows row_start[b] ..
row_start[b + 1] - 1 of the step and has kv_len[b] slots once they are
written; row i of its n rows sits at slot kv_len[b] - n + i, in page
pages[b, slot // page_size]. Rows behind the last sequence are padding and
stay as they were. The keys, values and queries are column ranges of the QKV
projection's rows (Q | K | V).

Head layouts are those of the package's workloads. Queries have a standard
deviation of 2, so that a softmax over thousands of slots has some slots that
count; keys and values are N(0, 1), stored as they come or as e4m3 codes with
one power of two per token and head.
"""
import math

import torch

own = False

# query heads, key/value heads, head dim
HEADS = {
    "neox160m": (12, 12, 64),
    "neox14b": (16, 16, 128),
    "qwen05b": (14, 2, 64),
    "qwen15b": (12, 2, 128),
    "qwen7b": (28, 4, 128),
    "tiny_qwen": (4, 2, 32),
}
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn}
BYTES = {"f32": 4, "bf16": 2, "e4m3": 1}


def _case(kind, heads, dtype, cache, page, B, rows, kv, single=0, window=0, pad=0, name=None):
    """B sequences of rows[0] .. rows[1] new tokens (`single` of them of one) and kv[0] .. kv[1] slots."""
    c = {"kind": kind, "heads": heads, "dtype": dtype, "cache": cache, "page": page, "B": B, "rows_lo": rows[0],
         "rows_hi": rows[1], "kv_lo": kv[0], "kv_hi": kv[1], "single": single, "window": window, "pad": pad}
    return dict(c, name=name) if name else c


def listed():
    return [
        # Decoding appends one token per sequence of a small batch: launch latency and little else.
        _case("write", "neox160m", "bf16", "bf16", 16, 8, (1, 1), (100, 1500), name="write_tokens"),
        # A prefill step of four prompts' chunks goes into 8-bit pages, and the values that later steps will see are
        # taken back for it (a program that attends with what it has stored).
        _case("write_read", "qwen7b", "bf16", "e4m3", 64, 4, (1800, 4100), (2000, 9000), pad=5,
              name="write_read_e4m3"),
        # A preempted sequence's 8-bit pages are taken out of the pool, widened, to be kept elsewhere.
        _case("read", "qwen7b", "bf16", "e4m3", 64, 4, (4000, 16001), (4000, 16001), name="read_e4m3"),
        # The same for a small fp32 model's cache, a few hundred slots.
        _case("read", "neox160m", "f32", "f32", 32, 2, (150, 333), (150, 333), name="read_f32"),
        # One user, one token, a short conversation: the smallest attention call.
        _case("attend", "qwen05b", "bf16", "bf16", 16, 1, (1, 1), (513, 513), name="token_small"),
        # A serving batch that decodes, conversations of very different lengths.
        _case("attend", "qwen7b", "bf16", "bf16", 64, 64, (1, 1), (60, 8100), name="tokens_b64"),
        # Long documents behind an 8-bit cache, a few sequences.
        _case("attend", "qwen7b", "bf16", "e4m3", 128, 9, (1, 1), (20000, 33000), name="tokens_long_e4m3"),
        # A prompt prefilled in chunks: one chunk of 512 tokens on what is there already.
        _case("attend", "qwen15b", "bf16", "bf16", 64, 1, (512, 512), (8192, 8192), name="chunk_512"),
        # The largest: two chunks of some thousand tokens over long contexts (MFMA bound).
        _case("attend", "qwen7b", "bf16", "bf16", 64, 2, (3900, 4096), (12000, 20000), name="chunk_long"),
        # A mixed step: most sequences decode, some bring chunks, 8-bit pages, padded to the captured batch.
        _case("attend", "qwen05b", "bf16", "e4m3", 32, 24, (100, 700), (300, 4096), single=18, pad=33,
              name="mixed_e4m3"),
        # Multi-head attention over a sliding window: chunks of ragged prompts.
        _case("attend", "neox14b", "bf16", "bf16", 16, 5, (150, 1027), (200, 6000), window=1024, name="chunk_window"),
        # Checking a converted model in fp32, a short chunk on a short context.
        _case("attend", "neox160m", "f32", "f32", 16, 2, (77, 200), (350, 1000), name="chunk_f32"),
    ]


def _lengths(case):
    """(rows, slots) of each sequence: spread over their ranges by the golden ratio, the same for every seed."""
    got = []
    for b in range(case["B"]):
        u, w = (0.5 + b * 0.6180339887) % 1.0, (0.5 + b * 0.7548776662) % 1.0
        n = 1 if b < case["single"] else round(case["rows_lo"] + u * (case["rows_hi"] - case["rows_lo"]))
        kv = round(case["kv_lo"] + w * (case["kv_hi"] - case["kv_lo"]))
        if case["kind"] == "read":
            n = kv  # the whole sequence
        got.append((n, max(kv, n)))
    return got


def work(case):
    hq, hkv, hd = HEADS[case["heads"]]
    eb, cb = BYTES[case["dtype"]], BYTES[case["cache"]]
    slot = 2 * hkv * (hd * cb + (1 if case["cache"] == "e4m3" else 0))  # a cached token's key and value
    row = 2 * hkv * hd * eb  # a new token's
    lens = _lengths(case)
    n = sum(r for r, _ in lens)
    if case["kind"] == "write":
        return {"bytes": n * (row + slot), "flops": 0}
    if case["kind"] == "read":
        return {"bytes": n * (row + slot), "flops": 0}
    if case["kind"] == "write_read":
        return {"bytes": n * 2 * (row + slot), "flops": 0}
    pairs = slots = 0
    w = case["window"] or 1 << 60
    for r, kv in lens:
        slots += min(kv, r - 1 + w)
        # row i sees min(kv - r + i + 1, w) slots
        first, full = kv - r + 1, max(0, min(r, w - (kv - r)))
        pairs += full * (2 * first + full - 1) // 2 + (r - full) * min(w, kv)
    return {"bytes": 2 * n * hq * hd * eb + slots * slot, "flops": 4 * hd * hq * pairs}


def _cost(case):
    """About what the case takes in seconds, to compare sizes."""
    w = work(case)
    return w["bytes"] / 3e12 + w["flops"] / (6e14 if case["dtype"] == "bf16" else 5e13)


def draw(rng):
    """One more call of the same ranges: decoding batches, chunks, mixed steps, and the cache's own traffic."""
    def log(lo, hi):
        return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))

    limit = max(_cost(c) for c in listed())
    while True:
        dtype, cache = rng.choice([("bf16", "bf16"), ("bf16", "bf16"), ("bf16", "e4m3"), ("bf16", "e4m3"),
                                   ("f32", "f32"), ("f32", "e4m3")])
        kind = rng.choice(["write", "write_read", "read", "attend", "attend", "attend", "attend", "attend"])
        if kind == "write":
            cache = dtype  # 8-bit codes are returned as the values they stand for: written and read back
        heads, page = rng.choice(sorted(HEADS)), rng.choice([16, 32, 64, 128, 256])
        kv = sorted((log(1, 24000), log(1, 24000)))
        shape = rng.choice(["tokens", "few", "chunk", "mixed"]) if kind == "attend" else "chunk"
        B = log(1, 96) if shape in ("tokens", "few") else log(1, 32)
        rows = sorted((log(1, 4096), log(1, 4096)))
        if shape == "tokens":
            rows = [1, 1]
        elif shape == "few":
            rows = [1, rng.randint(2, 9)]
        single = rng.randint(1, B) if shape == "mixed" else 0
        window = log(16, 4096) if kind == "attend" and rng.random() < 0.2 else 0
        pad = rng.choice([0, 0, rng.randint(1, 70)])
        c = _case(kind, heads, dtype, cache, page, B, rows, kv, single, window, pad)
        lens = _lengths(c)
        hq, hkv, hd = HEADS[heads]
        room = len(lens) * max(s for _, s in lens)  # slots of the padded batch
        scores = max(r for r, _ in lens) * room * hq
        if _cost(c) <= limit and scores <= 2.5e9 and room * hkv * hd <= 1.5e9:
            return c


def _pool(shape, cache, gen, dev):
    """A pool's pages as earlier sequences left them, and their exponents."""
    if cache != "e4m3":
        return torch.randn(shape, generator=gen, device=dev).to(DTYPES[cache]), None
    # a row's largest code is over 224; its power of two puts the values near N(0, 1)
    x = torch.randn(shape, generator=gen, device=dev).to(torch.bfloat16) * 128
    codes = x.float().clamp(-448, 448).to(torch.float8_e4m3fn)
    return codes, torch.randint(119, 122, shape[:-1], generator=gen, device=dev, dtype=torch.uint8)


def prepare(case, seed):
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev).manual_seed(int(seed))
    host = torch.Generator().manual_seed(int(seed))
    hq, hkv, hd = HEADS[case["heads"]]
    dt, page, B = DTYPES[case["dtype"]], case["page"], case["B"]
    lens = _lengths(case)
    lens = [lens[i] for i in torch.randperm(B, generator=host).tolist()]
    starts = [0]
    for r, _ in lens:
        starts.append(starts[-1] + r)
    n_rows = starts[-1] + case["pad"]
    held = [-(-kv // page) for _, kv in lens]
    max_pages, n_pages = max(held), sum(held) + 3
    order = torch.randperm(n_pages, generator=host).to(torch.int32)
    table = torch.zeros(B, max_pages, dtype=torch.int32)
    at = 0
    for b, m in enumerate(held):
        table[b, :m] = order[at:at + m]
        at += m
    k, k_exp = _pool((n_pages, hkv, page, hd), case["cache"], gen, dev)
    v, v_exp = _pool((n_pages, hkv, page, hd), case["cache"], gen, dev)
    st = {"case": case, "k": k, "v": v, "k_exp": k_exp, "v_exp": v_exp, "pages": table.to(dev),
          "row_start": torch.tensor(starts, dtype=torch.int32, device=dev),
          "kv_len": torch.tensor([kv for _, kv in lens], dtype=torch.int32, device=dev), "n_rows": n_rows,
          "max_rows": max(r for r, _ in lens)}
    if case["kind"] == "attend":
        qkv = torch.randn(n_rows, (hq + 2 * hkv) * hd, generator=gen, device=dev) * 2
        st["q"] = qkv.to(dt)[:, :hq * hd].view(n_rows, hq, hd)
        st["out"] = torch.zeros(n_rows, hq, hd, dtype=dt, device=dev)
    else:
        if case["kind"] != "read":
            qkv = torch.randn(n_rows, (hq + 2 * hkv) * hd, generator=gen, device=dev).to(dt)
            st["new_k"] = qkv[:, hq * hd:(hq + hkv) * hd].view(n_rows, hkv, hd)
            st["new_v"] = qkv[:, (hq + hkv) * hd:].view(n_rows, hkv, hd)
        if case["kind"] != "write":
            st["out_k"] = torch.zeros(n_rows, hkv, hd, dtype=dt, device=dev)
            st["out_v"] = torch.zeros(n_rows, hkv, hd, dtype=dt, device=dev)
    if own:  # the handles and the workspace that a serving program keeps
        import paper_2607_21291_amd as P
        st["cache"] = P.PagedCache(k, v, k_exp, v_exp)
        st["batch"] = P.PagedBatch(st["row_start"], st["kv_len"], st["pages"], n_rows, st["max_rows"])
        if case["kind"] == "attend":
            need = P.paged_attention_workspace_size(st["cache"], st["batch"], P.F32 if dt == torch.float32 else P.BF16, hq)
            st["workspace"] = torch.empty(max(need, 256), dtype=torch.uint8, device=dev)
    return st


def run(st):
    kind = st["case"]["kind"]
    if own:
        import paper_2607_21291_amd as P
        if kind == "attend":
            P.paged_attention(st["cache"], st["batch"], st["q"], st["out"], window=st["case"]["window"],
                              workspace=st["workspace"])
            return st["out"]
        if kind != "read":
            P.paged_cache_write(st["cache"], st["batch"], st["new_k"], st["new_v"])
        if kind == "write":
            return st["k"], st["v"]
        P.paged_cache_read(st["cache"], st["batch"], st["out_k"], st["out_v"])
        return st["out_k"], st["out_v"]
    if kind == "attend":
        return _attend(st)
    if kind != "read":
        _write(st, st["new_k"], st["k"], st["k_exp"])
        _write(st, st["new_v"], st["v"], st["v_exp"])
    if kind == "write":
        return st["k"], st["v"]
    return _read(st, st["k"], st["k_exp"], st["out_k"]), _read(st, st["v"], st["v_exp"], st["out_v"])


# ------------------------------------------------------------- plain forms

def _places(st):
    """Sequence, slot, page and place in the page of every row that a sequence has, and those rows."""
    start, B = st["row_start"].long(), st["case"]["B"]
    rows = torch.arange(st["n_rows"], device=start.device)
    seq = torch.searchsorted(start[1:], rows, right=True)
    rows, seq = rows[seq < B], seq[seq < B]
    slot = st["kv_len"].long()[seq] - (start[seq + 1] - rows)
    page = st["case"]["page"]
    return rows, seq, slot, st["pages"].long()[seq, slot // page], slot % page


def _two_to(e):
    """2^e in 32 bits for -126 <= e <= 127, from its bits (a power function may be off by its last bit)."""
    return ((e.int() + 127) << 23).view(torch.float32)


def _write(st, new, pool, exps):
    rows, _, _, page, place = _places(st)
    x = new[rows].float()
    if exps is None:
        pool[page, :, place] = x.to(pool.dtype)
        return
    # x / 448 = m 2^e with 1/2 <= m < 1: the least power of two with x <= 448 2^e is e, or e - 1 where m is 1/2
    top = x.abs().amax(-1)
    m, e = torch.frexp(top / 1.75)
    e = torch.where(m == 0.5, e - 1, e) - 8
    e = torch.where(top > 0, e, torch.full_like(e, -126)).clamp(-126, 120)
    codes = (x * _two_to(-e)[..., None]).to(torch.float8_e4m3fn)
    # as bytes, so that the assignment is an ordinary one
    pool.view(torch.uint8)[page, :, place] = codes.view(torch.uint8)
    exps[page, :, place] = (e + 127).to(torch.uint8)


def _widen(codes, exps):
    x = codes.float()
    return x if exps is None else x * _two_to(exps.int() - 127)[..., None]


def _read(st, pool, exps, like):
    rows, _, _, page, place = _places(st)
    if exps is None:
        x = pool[page, :, place].float()
    else:
        x = _widen(pool.view(torch.uint8)[page, :, place].view(pool.dtype), exps[page, :, place])
    out = torch.zeros_like(like)
    out[rows] = x.to(out.dtype)
    return out


def _attend(st):
    case = st["case"]
    hq, hkv, hd = HEADS[case["heads"]]
    B, page, n = case["B"], case["page"], st["max_rows"]
    tab = st["pages"].long()
    dev = tab.device

    def slots(pool, exps):  # [B, Hkv, slots, hd]
        if exps is None:
            x = pool[tab].float()
        else:
            x = _widen(pool.view(torch.uint8)[tab].view(pool.dtype), exps[tab])
        return x.transpose(1, 2).reshape(B, hkv, -1, hd)

    rows, seq, slot, _, _ = _places(st)
    place = rows - st["row_start"].long()[seq]
    q = torch.zeros(B, n, hq, hd, device=dev)
    at = torch.full((B, n), -1, device=dev)
    q[seq, place] = st["q"][rows].float()
    at[seq, place] = slot
    k = slots(st["k"], st["k_exp"])
    j = torch.arange(k.shape[2], device=dev)
    see = j <= at[..., None]  # [B, rows, slots]
    if case["window"]:
        see &= j > at[..., None] - case["window"]
    q = q.view(B, n, hkv, hq // hkv, hd).permute(0, 2, 3, 1, 4).reshape(B, hkv, -1, hd)
    s = torch.matmul(q, k.transpose(2, 3).contiguous()).div_(math.sqrt(hd))
    del k
    s = s.view(B, hkv, hq // hkv, n, -1).masked_fill_(~see[:, None, None], -math.inf)
    top = s.amax(-1, keepdim=True).clamp_min_(-3e38)
    s = s.sub_(top).exp_()
    total = s.sum(-1, keepdim=True)
    v = slots(st["v"], st["v_exp"])
    o = torch.matmul(s.view(B, hkv, -1, s.shape[-1]), v).view(B, hkv, hq // hkv, n, hd) / total.clamp_min_(1e-37)
    out = torch.zeros_like(st["out"])
    out[rows] = o.permute(0, 3, 1, 2, 4).reshape(B, n, hq, hd)[seq, place].to(out.dtype)
    return out


# ------------------------------------------- results in 64 bits, one sequence at a time

def _power(e):
    """2^e in 64 bits for whole e, from its bits."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _e4m3(x):
    """x (64 bits, at most 448) rounded to the nearest e4m3 number, ties to even: 3 fraction bits, least exponent -6."""
    _, e = torch.frexp(x.abs())  # below 2^e, and at least half of it
    step = _power((e - 1).clamp_min(-6) - 3)
    return torch.round(x / step) * step


def exact(case, seed):
    st = prepare(case, seed)
    hq, hkv, hd = HEADS[case["heads"]]
    page = case["page"]
    starts, kvs, pages = st["row_start"].tolist(), st["kv_len"].tolist(), st["pages"].long()

    def stored(pool, exps, b):  # the slots of sequence b: [slots, Hkv, hd]
        p = pages[b, :-(-kvs[b] // page)]
        if exps is None:
            x = pool[p].double()
        else:
            x = pool.view(torch.uint8)[p].view(pool.dtype).double() * _power(exps[p].long() - 127)[..., None]
        return x.permute(0, 2, 1, 3).reshape(-1, hkv, hd)[:kvs[b]]

    if case["kind"] == "write":
        outs = []
        for pool, new in ((st["k"], st["new_k"]), (st["v"], st["new_v"])):
            out = pool.double()
            for b in range(case["B"]):
                n = starts[b + 1] - starts[b]
                for h in range(hkv):
                    slot = torch.arange(kvs[b] - n, kvs[b], device=pool.device)
                    out[pages[b, slot // page], h, slot % page] = new[starts[b]:starts[b + 1], h].double()
            outs.append(out)
        return tuple(outs)
    if case["kind"] == "write_read":
        outs = []
        for new in (st["new_k"], st["new_v"]):
            x = new.double()
            if case["cache"] == "e4m3":
                top = x.abs().amax(-1, keepdim=True).clamp_min(2.0 ** -100)
                e = torch.ceil(torch.log2(top) - math.log2(448.0) - 1e-12)
                scale = _power(e)
                scale = torch.where(top > 448 * scale, scale * 2, scale)
                x = _e4m3(x / scale) * scale
            x[starts[-1]:] = 0
            outs.append(x)
        return tuple(outs)
    if case["kind"] == "read":
        outs = []
        for pool, exps in ((st["k"], st["k_exp"]), (st["v"], st["v_exp"])):
            out = torch.zeros(st["n_rows"], hkv, hd, dtype=torch.float64, device=pool.device)
            for b in range(case["B"]):
                n = starts[b + 1] - starts[b]
                out[starts[b]:starts[b + 1]] = stored(pool, exps, b)[kvs[b] - n:]
            outs.append(out)
        return tuple(outs)
    if work(case)["flops"] > 3e13:
        return None
    out = torch.zeros(st["n_rows"], hq, hd, dtype=torch.float64, device=pages.device)
    w = case["window"] or 1 << 40
    for b in range(case["B"]):
        k, v = stored(st["k"], st["k_exp"], b), stored(st["v"], st["v_exp"], b)
        n = starts[b + 1] - starts[b]
        i = torch.arange(kvs[b] - n, kvs[b], device=pages.device)[:, None]
        j = torch.arange(kvs[b], device=pages.device)
        hidden = (j > i) | (j <= i - w)
        for h in range(hq):
            q = st["q"][starts[b]:starts[b + 1], h].double()
            s = q @ k[:, h // (hq // hkv)].t().contiguous() * hd ** -0.5
            p = torch.softmax(s.masked_fill(hidden, -math.inf), -1)
            out[starts[b]:starts[b + 1], h] = p @ v[:, h // (hq // hkv)]
    return out
