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
