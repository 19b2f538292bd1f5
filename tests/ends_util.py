"""Inputs of the embedding, norm and head tests, and how far fp32 arithmetic may take their results from 64 bits.

u = 2^-24 is half a step of fp32 (each operation's relative error); sums in some order of length L are off by at most
L u times the sum of magnitudes. The matrix cores may drop instead of round: 2 u an addition there."""
import numpy as np
import torch

DT = {"f32": torch.float32, "bf16": torch.bfloat16}
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}  # half a step, relative
U = 2.0 ** -24
CODE = np.log(2.0) * 32 / 65535  # half a step of a logit's code (65535 to 64 factors of two), relative in a probability


def rand(shape, dtype, seed, scale=1.0, shift=0.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * scale + shift).to(DT[dtype])


def f64(t):
    return None if t is None else t.detach().cpu().double().numpy()


def close(got, want, bound, what=""):
    got, want = f64(got) if torch.is_tensor(got) else got, np.asarray(want)
    assert got.shape == want.shape
    bad = ~(np.abs(got - want) <= bound)
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.size} off, worst by {np.nanmax(np.abs(got - want) / bound):.3g} " \
                          f"of the bound, first at {np.argwhere(bad)[0]}"


def norm_bounds(x, w, b, eps, rms):
    """(bound on xh, relative bound on r, xh, r): the mean is a sum of d values (lanes of at most d / 64 + 8, then 10
    steps), subtracted once; the squares' sum as long; root, quotient and scaling 6 u."""
    d = x.shape[-1]
    L = d / 64 + 18
    m = 0.0 if rms else x.mean(-1, keepdims=True)
    dm = 0.0 if rms else (L + 2) * U * np.abs(x).mean(-1, keepdims=True)
    var = ((x - m) ** 2).mean(-1, keepdims=True)
    r = 1.0 / np.sqrt(var + eps)
    rr = (L + 4) * U + 6 * U + 2 * (dm * r) ** 2 + 2 * U * np.abs(m) * r
    xh = (x - m) * r
    return dm * r + np.abs(xh) * (rr + 4 * U) + 2 * U * np.abs(m) * r, rr, xh, r


def head_bounds(ref, h, w, dtype, half_out, dw_half):
    """Bounds on loss, dh and dw of a reference of ends_oracle.head.

    A logit is a sum of d products: chains of d / 32 additions of the matrix core's own sums of 32 (fp32: d / 2 of 2),
    scaled to log2 and by 1 / T: 4 u of itself. A dot product at a target is shorter. lse: the logits' error, exp2 and
    the sums (16 in a lane, 6 across lanes and waves, the tiles' in 16 chains and 16 more; fp32: V / 1024 and 16 more) and
    the logarithm's. p: those of z and lse, the code (bf16), 4 u. dz is rounded to dtype, in two terms where at most 128 rows take part
    (bf16). Products with dz: chains as
    above over classes or rows (plus 128 partial sums), then scale and rounding."""
    n, d = h.shape
    V, T, live = w.shape[0], ref["temperature"], ref["live"]
    h = np.where(live[:, None], h, 0.0)
    mag = np.abs(h) @ np.abs(w).T / T
    step = 32 if dtype == "bf16" else 2
    ez = (2 * (d / step + step) * U * mag + 6 * U * np.abs(ref["z"])).max(1)
    L = V / 4096 + 64 if dtype == "bf16" else V / 1024 + 64
    spread = np.abs(ref["z"]).max(1) + np.abs(ref["lse"])
    elogs = ez + L * U + 8 * U * (spread + 1)
    # sum q (lse - z) over a list: 16 chains and 16 more, q off by 64 u (its exponentials' sum over a list)
    k = 1 if ref["lists"] is None else ref["lists"]
    loss = T * T * ((ez + elogs + (64 + k / 16 + 24) * U * (spread + 1)) + (64 + k / 64 + 24) * U * (np.abs(ref["plogp"]) + 1))
    loss = (loss + HALF["f32"] * np.abs(ref["loss"])) * live
    rp = np.expm1((ez + elogs + 8 * U * (spread + 1)) + (CODE if dtype == "bf16" else 0.0))[:, None]
    wt = np.abs(ref["weight"])[:, None]
    edz = wt * (ref["p"] * rp + (0 if ref["lists"] is None else 64 * U) + 4 * U) * live[:, None]
    twin = dtype == "bf16" and live.sum() <= 128
    edz = edz + (HALF[dtype] ** 2 if twin else HALF[dtype]) * (np.abs(ref["dz"]) + edz)
    s = abs(ref["scale"])
    k1, k2 = V / step + step + (260 if twin else 130), (2 if twin else 1) * n / step + step + 4
    adz = np.abs(ref["dz"]) + edz
    dh = s * (edz @ np.abs(w) + 2 * k1 * U * (adz @ np.abs(w))) * (1 + 4 * U)
    dw = s * (edz.T @ np.abs(h) + 2 * k2 * U * (adz.T @ np.abs(h))) * (1 + 4 * U)
    dh = dh + half_out * (np.abs(ref["dh"]) + dh) + 1e-38
    dw = dw + dw_half * (np.abs(ref["dw"]) + dw) + 1e-38
    return loss, dh, dw
