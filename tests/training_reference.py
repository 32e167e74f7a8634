"""The operators around the step in 64 bits, from their definitions, with bounds on what 32-bit sums in any of the kernels' orders may be off:
u = 2^-24 per fp32 operation, half an ulp of the result's type for the last rounding, and (terms of the longest chain of additions) * u for a sum."""
import numpy as np
import torch

U = 2.0 ** -24
HALF_ULP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}
TINY = 1e-37          # results this small may be subnormal


def f64(t):
    return t.detach().double().cpu().numpy()


def within(got, ref, bound):
    """Whether |got - ref| <= bound everywhere; where ref is not finite, got is the same."""
    got = f64(got)
    assert got.shape == ref.shape, (got.shape, ref.shape)
    fine = np.isfinite(ref)
    assert np.array_equal(np.isnan(got), np.isnan(ref)) and np.array_equal(got[~fine & ~np.isnan(ref)], ref[~fine & ~np.isnan(ref)])
    over = np.abs(got - ref)[fine] - np.broadcast_to(bound, ref.shape)[fine]
    assert over.size == 0 or over.max() <= 0.0, f"over the bound by {over.max():.3e}, largest value {np.abs(ref[fine]).max():.3e}"


def embed_gradient(dout, ids, rows, scale, old, dtype):
    """-> (gradient, bound): sums over equal ids; old: what it is added to, or None."""
    dout, ids = f64(dout).reshape(-1, dout.shape[-1]), ids.cpu().numpy().reshape(-1)
    scale = float(np.float32(scale))
    keep = (ids >= 0) & (ids < rows)
    ref, size, terms = np.zeros((rows, dout.shape[1])), np.zeros((rows, dout.shape[1])), np.zeros((rows, 1))
    np.add.at(ref, ids[keep], dout[keep])
    np.add.at(size, ids[keep], np.abs(dout[keep]))
    np.add.at(terms, ids[keep], 1.0)
    ref, size = ref * scale, size * abs(scale)
    if old is not None:
        ref, size = ref + f64(old), size + np.abs(f64(old))
    return ref, (terms + 4) * U * size + HALF_ULP[dtype] * np.abs(ref) * (1 + 1e-3) + TINY


def chain(dim):
    return (dim // 64 + 24) * U


def layer_norm(x, w, b, eps, rms):
    """-> (y, bound of y, mean, bound, rstd, bound) for a matrix x."""
    dtype = x.dtype
    x = f64(x)
    dim = x.shape[1]
    w = np.ones(dim) if w is None else f64(w)
    b = np.zeros(dim) if b is None else f64(b)
    mean = np.zeros((len(x), 1)) if rms else x.mean(1, keepdims=True)
    off_mean = np.zeros((len(x), 1)) if rms else chain(dim) * np.abs(x).mean(1, keepdims=True) + U * np.abs(mean)
    d = x - mean
    off_d = off_mean + U * (np.abs(d) + off_mean)
    var = (d * d).mean(1, keepdims=True)
    # a shift of the mean by e moves the mean of (x - mu)^2 by e^2 only, the roundings of d by up to 2 |d| U |d|
    off_var = (chain(dim) + 4 * U) * var + 2 * off_mean ** 2 + 4 * U * off_mean * np.abs(d).mean(1, keepdims=True)
    eps = float(np.float32(eps))
    rstd = 1.0 / np.sqrt(var + eps)
    off_rstd = rstd * (0.5 * off_var / np.maximum(var + eps - off_var, 1e-300) + 6 * U)
    y = d * rstd * w + b
    off = np.abs(w) * (off_d * (rstd + off_rstd) + np.abs(d) * off_rstd) + 4 * U * (np.abs(d * rstd * w) + np.abs(b))
    return y, off + HALF_ULP[dtype] * (np.abs(y) + off) + TINY, mean[:, 0], off_mean[:, 0] + TINY, rstd[:, 0], off_rstd[:, 0]


def layer_norm_gradient(dy, x, w, mean, rstd, rms, old_dw, old_db, pdtype):
    """-> (dx, bound, dw, bound, db, bound) from the forward pass's fp32 mean and rstd."""
    dtype = x.dtype
    x, dy, r = f64(x), f64(dy), f64(rstd).reshape(-1, 1)
    mu = np.zeros_like(r) if rms else f64(mean).reshape(-1, 1)
    rows, dim = x.shape
    w = np.ones(dim) if w is None else f64(w)
    h, g = (x - mu) * r, dy * w
    s1 = np.zeros_like(r) if rms else g.mean(1, keepdims=True)
    s2 = (g * h).mean(1, keepdims=True)
    off1 = 0.0 if rms else (chain(dim) + U) * np.abs(g).mean(1, keepdims=True)
    off2 = (chain(dim) + 4 * U) * np.abs(g * h).mean(1, keepdims=True)
    dx = r * (g - s1 - h * s2)
    off = np.abs(r) * (6 * U * (np.abs(g) + np.abs(s1) + np.abs(h * s2)) + off1 + np.abs(h) * off2)
    long = (rows / 4 + 64) * U
    out = [dx, off + HALF_ULP[dtype] * (np.abs(dx) + off) + TINY]
    for per_row, old in ((dy * h, old_dw), (dy, old_db)):
        ref, size = per_row.sum(0), np.abs(per_row).sum(0)
        if old is not None:
            ref, size = ref + f64(old), size + np.abs(f64(old))
        o = (long + 4 * U) * size
        out += [ref, o + HALF_ULP[pdtype] * (np.abs(ref) + o) + TINY]
    return out
