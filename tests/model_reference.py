"""AdamW, rotary positions and the block norm in 64 bits, from their definitions in include/fira.h, with bounds on what fp32 may be off: u = 2^-24
for each operation in fp32, half an ulp of the result's type for its rounding (training_reference.py)."""
import math

import numpy as np
import torch

from training_reference import HALF_ULP, TINY, U, chain, f64

MASK = 0xFFFFFFFF


# ---- AdamW ---------------------------------------------------------------------------------------------------------


def mix(x):
    x = np.asarray(x, dtype=np.uint64) & np.uint64(MASK)
    x ^= x >> np.uint64(16)
    x = (x * np.uint64(0x6A09E667)) & np.uint64(MASK)
    x ^= x >> np.uint64(15)
    x = (x * np.uint64(0xBB67AE85)) & np.uint64(MASK)
    return x ^ (x >> np.uint64(16))


def rounding(n, seed, t, first=0):
    """The 16-bit numbers that m and sqrt(v) of values first .. first + n of a tensor are rounded by in step t."""
    key = mix(mix(seed) + np.uint64(t & MASK))
    h = mix(np.arange(first, first + n, dtype=np.uint64) + key)
    return h & np.uint64(0xFFFF), h >> np.uint64(16)


def e4m3(codes):
    """Values of a float8_e4m3fn tensor, from its bits."""
    b = codes.detach().reshape(-1).view(torch.uint8).cpu().numpy().astype(np.int64)
    exponent, mantissa = b >> 3 & 15, b & 7
    x = np.where(exponent == 0, mantissa * 2.0 ** -9, (8 + mantissa) * 2.0 ** (exponent - 10.0))
    return np.where(b & 127 == 127, np.nan, np.where(b & 128, -x, x))


def block_most(x):
    """Largest finite size of each block of 256 values, for each value's place and for the blocks."""
    size = np.where(np.isfinite(x), np.abs(x), 0.0)
    blocks = np.pad(size, (0, -len(x) % 256)).reshape(-1, 256).max(1)
    return np.repeat(blocks, 256)[:len(x)], blocks


def held(x, most, random, floor, off):
    """What is held of sizes x, in units of the scale, if x * 448 / most came out off by the factor 1 + off."""
    with np.errstate(invalid="ignore", divide="ignore"):
        y = np.minimum(np.abs(x) * (448.0 / most) * (1.0 + off), 448.0)
        step = 2.0 ** (np.floor(np.log2(np.maximum(y, 2.0 ** -6))) - 3.0)
        c = np.minimum(np.floor(y / step + (random.astype(np.float64) + 0.5) / 65536.0) * step, 448.0)
    if floor:
        c = np.where(y > 0.0, np.maximum(c, 2.0 ** -9), c)
    return np.where(np.isfinite(x), c, np.nan)


def adamw(w, g, m, v, taken, decay, lr, b1, b2, eps, cut=1.0):
    """-> {name: (value, bound)} of w, m, v and sqrt(v) after a step; all arrays of fp64, m and v the fp32 values they were read as (v of 8 bits: a root, squared in
    fp32).  Roundings counted one by one: the betas and 1 - beta in fp32, the cut and its product, each product and sum."""
    t = taken + 1
    g = g * cut
    m2, off_m = b1 * m + (1 - b1) * g, 6 * U * (np.abs(b1 * m) + np.abs((1 - b1) * g))
    v2, off_v = b2 * v + (1 - b2) * g * g, 10 * U * (b2 * v + (1 - b2) * g * g)
    root = np.sqrt(v2)
    off_root = 6 * U * root
    k1, k2 = 1.0 / (1.0 - b1 ** t), 1.0 / math.sqrt(1.0 - b2 ** t)
    below = root * k2 + eps
    step = lr * k1 * m2 / below
    off = lr * k1 * off_m / below + 14 * U * np.abs(step)
    w2 = w * (1.0 - lr * decay) - step
    # (the smallest results are fp32 subnormals: off by a step of those)
    return {"w": (w2, off + 3 * U * np.abs(w) + U * np.abs(step)), "m": (m2, off_m + 1e-44), "v": (v2, off_v + 1e-44), "root": (root, off_root + 1e-22)}


# ---- rotary positions ----------------------------------------------------------------------------------------------


def rotary(x, positions, frequencies, interleaved, scale, gradient):
    """x: (batch, length, heads, dim), positions: (batch, length) whole numbers -> (y, bound).  Off may be: the angle by 4 roundings of fp64 and one of fp32 of half a turn, the sine by
    4 u, its scale by 1, products and sum by 3."""
    dtype = x.dtype
    x, f = f64(x), f64(frequencies)
    scale = float(np.float32(scale))
    angle = np.asarray(positions, dtype=np.float64)[..., None] * f
    off_angle = (np.abs(angle) * 4 * 2.0 ** -53 + math.pi * U + 5 * U)[..., None, :]
    c, s = scale * np.cos(angle)[..., None, :], scale * (-np.sin(angle) if gradient else np.sin(angle))[..., None, :]
    half, rotated = len(f), 2 * len(f)
    a, b = (slice(0, rotated, 2), slice(1, rotated, 2)) if interleaved else (slice(0, half), slice(half, rotated))
    y, off = x.copy(), np.zeros_like(x)
    y[..., a], y[..., b] = x[..., a] * c - x[..., b] * s, x[..., a] * s + x[..., b] * c
    size = abs(scale) * (np.abs(x[..., a]) + np.abs(x[..., b])) * (off_angle + 3 * U)
    off[..., a] = off[..., b] = size
    return y, off + np.where(off > 0, HALF_ULP[dtype] * (np.abs(y) + off) * (1 + 1e-3) + TINY, 0.0)


# ---- block norm ----------------------------------------------------------------------------------------------------


def _vector(v, dim, default):
    return np.full(dim, default) if v is None else f64(v)


def normed(x, off_x, w, b, eps, kind):
    """Norm of fp64 rows that are off by up to off_x -> (y, off), (mean, off), (rstd, off); kind: "layer", "rms", "none"."""
    if kind == "none":
        return (x, off_x), None, None
    dim = x.shape[1]
    mean, off_mean = np.zeros((len(x), 1)), np.zeros((len(x), 1))
    if kind == "layer":
        mean = x.mean(1, keepdims=True)
        off_mean = chain(dim) * np.abs(x).mean(1, keepdims=True) + U * np.abs(mean) + off_x.mean(1, keepdims=True)
    d = x - mean
    off_d = off_x + off_mean + U * (np.abs(d) + off_mean)
    var = (d * d).mean(1, keepdims=True)
    off_var = (chain(dim) + 4 * U) * var + 2 * (np.abs(d) * off_d).mean(1, keepdims=True) + (off_d ** 2).mean(1, keepdims=True)
    eps = float(np.float32(eps))
    rstd = 1.0 / np.sqrt(var + eps)
    off_rstd = rstd * (0.5 * off_var / np.maximum(var + eps - off_var, 1e-300) + 6 * U)
    y = d * rstd * w + b
    off = np.abs(w) * (off_d * (rstd + off_rstd) + np.abs(d) * off_rstd) + 4 * U * (np.abs(d * rstd * w) + np.abs(b))
    return (y, off), (mean[:, 0], off_mean[:, 0] + TINY), (rstd[:, 0], off_rstd[:, 0])


def rounded(x, off, dtype):
    return x, off + HALF_ULP[dtype] * (np.abs(x) + off) + TINY


def block_norm(x, block, v, norm, post, eps, post_eps, beta, alpha):
    """v: dict of gate, weight, bias, post_weight, post_bias -> [(value, bound) of residual, y, mean, rstd, post_mean, post_rstd, or None]."""
    dtype, dim = x.dtype, x.shape[1]
    beta, alpha = float(np.float32(beta)), float(np.float32(alpha))
    x, b = f64(x), f64(block)
    (u, off), pm, ps = normed(b, np.zeros_like(b), _vector(v["post_weight"], dim, 1.0), _vector(v["post_bias"], dim, 0.0), post_eps, post)
    gate = _vector(v["gate"], dim, 1.0)
    u, off = gate * u, np.abs(gate) * off + U * np.abs(gate * u)
    r = beta * x + alpha * u
    off = abs(alpha) * off + 3 * U * (np.abs(beta * x) + np.abs(alpha * u))
    (y, off_y), mean, rstd = normed(r, off, _vector(v["weight"], dim, 1.0), _vector(v["bias"], dim, 0.0), eps, norm)
    of = lambda s, kind: s if kind == "layer" else None  # noqa: E731
    return [rounded(r, off, dtype), rounded(y, off_y, dtype) if norm != "none" else None, of(mean, norm), rstd, of(pm, post), ps]


def block_norm_gradient(dr, dy, r, block, v, stats, norm, post, beta, alpha, old, pdtype):
    """stats: mean, rstd, post_mean, post_rstd; old: what each vector's gradient is added to, or None -> [(value, bound) of dx, dblock] and a dict of those of
    gate, weight, bias, post_weight, post_bias."""
    dtype, (rows, dim) = r.dtype, r.shape
    beta, alpha = float(np.float32(beta)), float(np.float32(alpha))
    long = (rows / 4 + 64) * U
    r, b = f64(r), f64(block)
    column = lambda s, wanted, other: f64(s).reshape(-1, 1) if wanted else np.full((rows, 1), other)  # noqa: E731
    mu, rs = column(stats[0], norm == "layer", 0.0), column(stats[1], norm != "none", 1.0)
    pm, ps = column(stats[2], post == "layer", 0.0), column(stats[3], post != "none", 1.0)
    t = np.zeros_like(r) if dr is None else f64(dr)
    off_t = np.zeros_like(r)
    sums = {}
    if norm != "none":
        w, dy = _vector(v["weight"], dim, 1.0), f64(dy)
        h, g = (r - mu) * rs, dy * w
        s1 = g.mean(1, keepdims=True) if norm == "layer" else np.zeros((rows, 1))
        s2 = (g * h).mean(1, keepdims=True)
        off1 = (chain(dim) + 2 * U) * np.abs(g).mean(1, keepdims=True) if norm == "layer" else 0.0
        off2 = (chain(dim) + 6 * U) * np.abs(g * h).mean(1, keepdims=True)
        off_t = np.abs(rs) * (6 * U * (np.abs(g) + np.abs(s1) + np.abs(h * s2)) + off1 + np.abs(h) * off2)
        added = rs * (g - s1 - h * s2)
        off_t = off_t + 2 * U * (np.abs(t) + np.abs(added))
        t = t + added
        sums["weight"] = ((dy * h).sum(0), (long + 6 * U) * np.abs(dy * h).sum(0))
        sums["bias"] = (dy.sum(0), (long + 6 * U) * np.abs(dy).sum(0))
    gate, pw, pb = _vector(v["gate"], dim, 1.0), _vector(v["post_weight"], dim, 1.0), _vector(v["post_bias"], dim, 0.0)
    hb = (b - pm) * ps
    q0 = alpha * gate * t
    q = q0 * pw
    off_q = np.abs(alpha * gate * pw) * off_t + 4 * U * np.abs(q)
    if post != "none":
        q1 = q.mean(1, keepdims=True) if post == "layer" else np.zeros((rows, 1))
        q2 = (q * hb).mean(1, keepdims=True)
        off1 = (chain(dim) + 2 * U) * np.abs(q).mean(1, keepdims=True) + off_q.mean(1, keepdims=True) if post == "layer" else 0.0
        off2 = (chain(dim) + 6 * U) * np.abs(q * hb).mean(1, keepdims=True) + (off_q * np.abs(hb)).mean(1, keepdims=True)
        db = ps * (q - q1 - hb * q2)
        off_db = np.abs(ps) * (6 * U * (np.abs(q) + np.abs(q1) + np.abs(hb * q2)) + off_q + off1 + np.abs(hb) * off2)
    else:
        db, off_db = q, off_q
    s2, off2 = (t * hb).sum(0), (long + 6 * U) * np.abs(t * hb).sum(0) + (off_t * np.abs(hb)).sum(0)
    s3, off3 = t.sum(0), (long + 6 * U) * np.abs(t).sum(0) + off_t.sum(0)
    sums["gate"] = (alpha * (pw * s2 + pb * s3), abs(alpha) * (np.abs(pw) * off2 + np.abs(pb) * off3 + 4 * U * (np.abs(pw * s2) + np.abs(pb * s3))))
    sums["post_weight"] = (alpha * gate * s2, np.abs(alpha * gate) * (off2 + 4 * U * np.abs(s2)))
    sums["post_bias"] = (alpha * gate * s3, np.abs(alpha * gate) * (off3 + 4 * U * np.abs(s3)))
    for k, (x, off) in sums.items():
        if old is not None and old.get(k) is not None:
            before = f64(old[k])
            x, off = x + before, off + 2 * U * (np.abs(x) + np.abs(before))
        sums[k] = rounded(x, off, pdtype)
    return [rounded(beta * t, abs(beta) * off_t + 2 * U * np.abs(beta * t), dtype), rounded(db, off_db, dtype)], sums
